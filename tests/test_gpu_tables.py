"""Page tables of a cache built on the GPU, against the definition sequence by sequence on the host."""
import math
import random

import pytest
import torch

from cache_cases import dequantise, quantise

pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(scope="module")
def heart():
    from paper_2605_14513_b200 import heart as h

    return h


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


class Tables:
    """A list of free pages and the sequences' tables, on the host and on the GPU."""

    def __init__(self, heart, lens, page=16, T=64, n_pages=None, spare=40, width=None, seed=0):
        rng = random.Random(seed)
        self.heart, self.page, self.S, self.T = heart, page, len(lens), T
        held = [-(-n // page) for n in lens]
        self.n_pages = n_pages or sum(held) + spare
        self.width = width or max(held + [1]) + 8
        order = list(range(self.n_pages))
        rng.shuffle(order)
        self.table = [[-7] * self.width for _ in lens]
        at = 0
        for row, n in zip(self.table, held):
            row[:n] = order[at:at + n]
            at += n
        self.count = self.n_pages - at
        self.free = order[at:] + [-9] * at
        self.lens, self.row_start = list(lens), [0] * (self.S + 1)
        self.cfg = heart.make_cache_config(self.S, T, 2, 2, page, self.n_pages, self.width)
        self.ws = heart.new_cache_workspace(self.cfg)
        self.d = dict(kv_len=ints(self.lens), free_pages=ints(self.free), free_count=ints([self.count]), page_table=ints(self.table))
        self.d_row_start, self.d_slots = ints([5] * (self.S + 1)), ints([-3] * T, torch.int64)

    # the definition, on the host
    def extend(self, new):
        self.row_start, self.slots = [0], []
        for s, n in enumerate(new):
            for j in range(-(-self.lens[s] // self.page), -(-(self.lens[s] + n) // self.page)):
                self.count -= 1
                self.table[s][j] = self.free[self.count]
            self.slots += [self.table[s][p // self.page] * self.page + p % self.page for p in range(self.lens[s], self.lens[s] + n)]
            self.lens[s] += n
            self.row_start.append(self.row_start[-1] + n)
        self.slots += [-1] * (self.T - len(self.slots))

    def release(self, ended):
        for s, e in enumerate(ended):
            if e:
                n = -(-self.lens[s] // self.page)
                self.free[self.count:self.count + n] = self.table[s][:n]
                self.count += n
                self.lens[s] = 0

    # the calls
    def run_extend(self, new, slots=True, **out):
        self.heart.heart_cache_extend(self.cfg, ints(new), ws=self.ws, row_start=self.d_row_start, slots=self.d_slots if slots else None, **self.d, **out)

    def run_release(self, ended, **out):
        self.heart.heart_cache_release(self.cfg, ints(ended, torch.uint8), ws=self.ws, **self.d, **out)

    def check(self, slots=True, rows=True):
        assert self.d["kv_len"].tolist() == self.lens and self.d["free_count"].tolist() == [self.count]
        assert self.d["page_table"].tolist() == self.table and self.d["free_pages"].tolist() == self.free
        if rows:
            assert self.d_row_start.tolist() == self.row_start
        if slots and rows:
            assert self.d_slots.tolist() == self.slots
        return self.heart.heart_get_status(self.ws)


CASES = {
    "one": dict(lens=[0], new=[1]),
    "nothing": dict(lens=[5], new=[0]),
    "a page to its end": dict(lens=[15, 16, 17], new=[1, 1, 15]),
    "over an end": dict(lens=[15, 16, 1], new=[2, 16, 33], page=16),
    "prompts and tokens": dict(lens=[0, 100, 3, 0], new=[130, 1, 0, 17], page=32, T=200),
    "pages of 128": dict(lens=[127, 128, 0], new=[1, 1, 300], page=128, T=302),
    "all rows": dict(lens=[1, 2], new=[30, 34], T=64),
    "33 sequences": dict(lens=list(range(33)), new=[(i * 5) % 7 for i in range(33)], T=150),
    "1024 sequences": dict(lens=[(i * 37) % 90 for i in range(1024)], new=[(i * 11) % 5 for i in range(1024)], T=5000, spare=2000),
    "1025 sequences": dict(lens=[(i * 37) % 90 for i in range(1025)], new=[(i * 11) % 5 for i in range(1025)], T=5000, spare=2000),
    "2500 sequences": dict(lens=[(i * 31) % 50 for i in range(2500)], new=[(i * 13) % 9 for i in range(2500)], T=12000, spare=5000),
    "a long prompt": dict(lens=[3, 7], new=[20000, 1], T=20100, spare=1300, width=1300),
}


@pytest.mark.parametrize("name", CASES)
def test_extend(heart, name):
    kw = dict(CASES[name])
    new = kw.pop("new")
    t = Tables(heart, **kw)
    t.run_extend(new)
    t.extend(new)
    assert t.check() == 0
    # without slots, and apart from the lengths and the count before
    u = Tables(heart, **kw)
    u.run_extend(new, slots=False, kv_len_out=(lens := ints([0] * u.S)), free_count_out=(count := ints([0])))
    assert u.d["kv_len"].tolist() == u.lens and u.d["free_count"].tolist() == [u.count]
    assert lens.tolist() == t.lens and count.tolist() == [t.count] and u.d["page_table"].tolist() == t.table
    assert u.d_row_start.tolist() == t.row_start and (u.d_slots == -3).all()
    # the same call again gives the same: nothing that it reads has changed
    u.run_extend(new, kv_len_out=lens, free_count_out=count)
    assert lens.tolist() == t.lens and u.d_slots.tolist() == t.slots and heart.heart_get_status(u.ws) == 0


@pytest.mark.parametrize("name", CASES)
def test_release(heart, name):
    kw = dict(CASES[name])
    kw.pop("new")
    for part in (2, 1):
        ended = [int(s % part == 0) * (1 + s % 3) for s in range(len(kw["lens"]))]  # (anything but 0)
        t = Tables(heart, **kw)
        t.run_release(ended)
        t.release(ended)
        assert t.check(rows=False) == 0
        u = Tables(heart, **kw)
        u.run_release(ended, kv_len_out=(lens := ints([9] * u.S)), free_count_out=(count := ints([0])))
        assert u.d["kv_len"].tolist() == u.lens and lens.tolist() == t.lens and count.tolist() == [t.count]
        assert u.d["free_pages"].tolist() == t.free and u.d["page_table"].tolist() == t.table


def test_calls_that_cannot_be_done(heart):
    """Nothing changes, the rows are none, the status tells."""
    big = (1 << 31) - 1
    for S in (3, 1030):
        fill = [0] * (S - 3)
        for lens, new, kw in (([5, 0, 3], [60, 5, 0], {}), ([5, 0, 3], [1, -1, 2], {}), ([5, 0, 3], [1, big, big], {}), ([0, 0, 0], [20, 20, 20], dict(n_pages=5)),
                              ([0, 0, 0], [17, 1, 1], dict(width=1)), ([0, 1, 0], [big, 0, 0], {})):
            for out in (False, True):
                for slots in (True, False):
                    t = Tables(heart, lens + fill, **{"spare": 50, **kw})
                    o = dict(kv_len_out=ints([1] * S), free_count_out=ints([1])) if out else {}
                    t.run_extend(new + fill, slots=slots, **o)
                    t.row_start, t.slots = [0] * (S + 1), [-1] * t.T
                    assert t.check(slots=slots) == heart.ERR_DEVICE_CHECK
                    if out:
                        assert o["kv_len_out"].tolist() == t.lens and o["free_count_out"].tolist() == [t.count]
    for bad in ("length", "negative length", "count", "negative count"):
        t = Tables(heart, [5, 40, 3])
        if bad == "length":
            t.lens[1] = t.width * t.page + 1
        elif bad == "negative length":
            t.lens[1] = -1
        else:
            t.count = t.n_pages + 1 if bad == "count" else -1
        t.d["kv_len"].copy_(ints(t.lens))
        t.d["free_count"].fill_(t.count)
        t.run_extend([1, 0, 1])
        t.row_start, t.slots = [0] * 4, [-1] * t.T
        assert t.check() == heart.ERR_DEVICE_CHECK
        t.run_release([1, 1, 1])
        assert t.check() == heart.ERR_DEVICE_CHECK
        t.run_release([1, 0, 1])
        if "count" in bad:
            assert t.check() == heart.ERR_DEVICE_CHECK
        else:  # the length of a sequence that goes on is not looked at
            t.release([1, 0, 1])
            assert t.check() == 0
    t = Tables(heart, [16 * 5] * 3, spare=4)  # (more pages back than there are: a sequence ended twice)
    t.count = 8
    t.d["free_count"].fill_(8)
    t.run_release([1, 1, 1])
    assert t.check(rows=False) == heart.ERR_DEVICE_CHECK


def test_a_captured_step_goes_on_from_the_last(heart):
    """extend and release captured once, replayed with other lengths: requests come, grow and go, and no page is in two places."""
    rng = random.Random(4)
    S, page = 70, 16
    t = Tables(heart, [0] * S, page=page, T=3000, n_pages=3000, width=300)
    new, ended = ints([0] * S), ints([0] * S, torch.uint8)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        heart.heart_cache_release(t.cfg, ended, ws=t.ws, **t.d)
        heart.heart_cache_extend(t.cfg, new, ws=t.ws, row_start=t.d_row_start, slots=t.d_slots, **t.d)
    for step in range(30):
        e = [int(rng.random() < 0.1) for _ in range(S)]
        n = [rng.choice([0, 1, 1, 1, rng.randint(2, 200)]) if rng.random() < 0.5 or not e[s] else 0 for s in range(S)]
        while sum(n) > t.T:
            n[rng.randrange(S)] = 0
        ended.copy_(ints(e, torch.uint8))
        new.copy_(ints(n))
        graph.replay()
        torch.cuda.synchronize()
        t.release(e)
        t.extend(n)
        assert t.check() == 0
        live = [p for s in range(S) for p in t.table[s][:-(-t.lens[s] // page)]] + t.free[:t.count]
        assert sorted(live) == list(range(t.n_pages))


def test_more_than_a_launchs_ctas_of_rows(heart):
    """A launch of all CTAs, in place: 400 000 rows."""
    S = 100
    t = Tables(heart, [(s * 77) % 1000 for s in range(S)], T=410000, n_pages=40000, width=400)
    new = [4000 + (s % 7) for s in range(S)]
    t.run_extend(new)
    t.extend(new)
    assert t.check() == 0
    t.run_release([s % 2 for s in range(S)])
    t.release([s % 2 for s in range(S)])
    assert t.check(rows=False) == 0


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_run_of_a_models_steps(heart, kind):
    """Requests come, their chunks are given pages, written, attended to over the cache and then to a text of each request's own, and they go: every call on the
    arrays that the tables' calls have made, and the results against 64 bits."""
    rng = random.Random(9)
    g = torch.Generator().manual_seed(9)
    S, H, page, T = 3, 2, 16, 96
    n_pages, width = 40, 12
    texts = [40, 0, 130]
    states = [torch.randn((sum(texts), H, D), generator=g).to(torch.bfloat16) for _ in range(2)]
    starts = [0, 40, 40]
    cfg = heart.make_cache_config(S, T, H, H, page, n_pages, width, kind=heart.CACHE_E4M3 if kind == "e4m3" else heart.CACHE_BF16, causal=1)
    cross = heart.make_cross_config(S, T, sum(texts), H, H)
    cache, ws, cross_ws = heart.Cache(cfg), heart.new_cache_workspace(cfg), heart.new_cross_workspace(cross)
    free_pages = ints(list(range(n_pages)))
    free_count, kv_len, row_start = ints([n_pages]), ints([0] * S), ints([0] * (S + 1))
    table = torch.zeros((S, width), dtype=torch.int32, device="cuda")
    kept = [[torch.zeros((0, H, D), dtype=torch.bfloat16)] * 2 for _ in range(S)]
    dK, dV = (x.cuda() for x in states)
    k_start, k_len = ints(starts), ints(texts)
    for step in range(8):
        ended = [int(len(kept[s][0]) > 60) for s in range(S)]
        new = [rng.choice([1, 1, 20, 37]) if rng.random() < 0.8 else 0 for _ in range(S)]
        Q, K, V = (torch.randn((T, H, D), generator=g).to(torch.bfloat16) for _ in range(3))
        heart.heart_cache_release(cfg, ints(ended, torch.uint8), kv_len, free_pages, free_count, table, ws)
        heart.heart_cache_extend(cfg, ints(new), kv_len, free_pages, free_count, table, row_start, ws)
        O, P = (torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        heart.heart_cache_write(cfg, K.cuda(), V.cuda(), cache, table, row_start, kv_len, ws)
        heart.heart_cache_attn(cfg, Q.cuda(), cache, table, row_start, kv_len, O, ws)
        heart.heart_cross_attn(cross, O, dK, dV, row_start, k_start, k_len, P, cross_ws)
        assert heart.heart_get_status(ws) == 0 and heart.heart_get_status(cross_ws) == 0
        at = 0
        for s in range(S):
            n = new[s]
            kept[s] = [torch.cat([x[:0] if ended[s] else x, y[at:at + n]]) for x, y in zip(kept[s], (K, V))]
            L = len(kept[s][0])
            assert int(kv_len[s]) == L
            if n:
                k, v = ((dequantise(*quantise(x)) if kind == "e4m3" else x.double()).transpose(0, 1) for x in kept[s])
                logits = Q[at:at + n].double().transpose(0, 1) @ k.transpose(1, 2) / math.sqrt(D)
                logits.masked_fill_(torch.arange(L)[None] > torch.arange(L - n, L)[:, None], -math.inf)
                want = (torch.softmax(logits, -1) @ v).transpose(0, 1)
                got = O[at:at + n].cpu().double()
                # (weights and the result rounded once each, 2^-8; |v| below 5)
                assert ((got - want).abs() <= 2 ** -8 * want.abs() + 2 ** -8 * 5).all()
                # the cross attention takes what the cached one gave
                if texts[s]:
                    k, v = (x[starts[s]:starts[s] + texts[s]].double().transpose(0, 1) for x in states)
                    want = (torch.softmax(got.transpose(0, 1) @ k.transpose(1, 2) / math.sqrt(D), -1) @ v).transpose(0, 1)
                    assert ((P[at:at + n].cpu().double() - want).abs() <= 2 ** -8 * want.abs() + 2 ** -8 * 5).all()
                else:
                    assert (P[at:at + n] == 0).all()
            at += n
        assert (O[at:] == 0).all() and (P[at:] == 0).all()
    held = [p for s in range(S) for p in table[s, :-(-int(kv_len[s]) // page)].tolist()]
    assert sorted(held + free_pages[:int(free_count)].tolist()) == list(range(n_pages))


def test_wrong_tensors_are_refused(heart):
    t = Tables(heart, [5, 20])
    new, ended, n = ints([1, 1]), ints([0, 1], torch.uint8), t.n_pages
    good = dict(t.d, row_start=t.d_row_start, ws=t.ws)
    heart.heart_cache_extend(t.cfg, new, **good)
    for kw in (dict(new_len=new.long()), dict(new_len=new[:1]), dict(new_len=new.cpu()), dict(kv_len=ints([1])), dict(free_pages=ints([0] * (n - 1))),
               dict(free_count=ints([1, 2])), dict(page_table=good["page_table"].t()), dict(row_start=new), dict(slots=ints([0] * t.T)),
               dict(slots=ints([0] * (t.T + 1), torch.int64)), dict(kv_len_out=ints([0])), dict(free_count_out=ints([0], torch.int64)), dict(ws=t.ws[:512]),
               dict(ws=t.ws.cpu())):
        with pytest.raises(ValueError):
            heart.heart_cache_extend(t.cfg, **{"new_len": new, **good, **kw})
    for kw in (dict(ended=ended.bool()), dict(ended=ended[:1]), dict(kv_len=ints([1])), dict(free_pages=ints([0] * (n - 1))), dict(kv_len_out=ints([0])), dict(ws=t.ws.cpu())):
        with pytest.raises(ValueError):
            heart.heart_cache_release(t.cfg, **{"ended": ended, **t.d, "ws": t.ws, **kw})
