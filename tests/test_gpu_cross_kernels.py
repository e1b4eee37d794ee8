"""Cross attention on the GPU, every kernel where it can go wrong.  Which kernel a call takes is asked of the test-hook build, so that a rule that changes does not
lead these cases elsewhere unseen."""
import ctypes as C
import math

import pytest
import torch

from test_gpu_cross import Case, Device, heart, same  # noqa: F401  (heart: a fixture)

pytestmark = pytest.mark.gpu

D = 128
ROWS8, ROWS16, TILES, PAIRS = range(4)  # as CrossKernel has them
FAR = 70000  # rows of keys behind the sequences', times two key heads: more than L2 keeps, where pairs of CTAs begin


@pytest.fixture(scope="module")
def kernel_of():
    from paper_2605_14513_b200 import build

    lib = C.CDLL(build.build_test_hooks())
    return lambda cfg: lib.heart_test_cross_kernel(C.byref(cfg))


def exact(c, of):
    """The definition in 64 bits for the sequences (first row, rows, first key, keys): O, lse, sum_j w_j |v_j| and the largest sum of a logit's magnitudes."""
    O, B = torch.zeros((c.T, c.Hq, D), dtype=torch.float64), torch.zeros((c.T, c.Hq, D), dtype=torch.float64)
    lse = torch.full((c.T, c.Hq), -math.inf, dtype=torch.float64)
    scale, size = c.scale if c.scale > 0 else 1 / math.sqrt(D), 1.0
    for r0, n, f, L in of:
        for h in range(c.Hq if n and L else 0):
            q = c.Q[r0:r0 + n, h].double()
            k, v = (x[f:f + L, h // (c.Hq // c.Hkv)].double() for x in (c.K, c.V))
            logits = q @ k.T * scale
            size = max(size, float((q.abs() @ k.abs().T).max()) * scale)
            lse[r0:r0 + n, h] = torch.logsumexp(logits, -1)
            w = torch.softmax(logits, -1)
            O[r0:r0 + n, h], B[r0:r0 + n, h] = w @ v, w @ v.abs()
    return O, lse, B, size


def near(c, of, rows, O, lse):
    """The rows are what the definition says.  A logit is the sum of eight products of 16 dims, each rounded by 2^-23 of the magnitudes at most, times the scale (2^-23 with
    its factor's own rounding): off by 10 x 2^-23 of them.  Weights and their sum are off by as much each, a weight for the product by 2^-8 more, the result by 2^-8; sums of
    32-bit numbers 2^-12 in all."""
    want, want_lse, weights, size = exact(c, of)
    off = 10 * 2 ** -23 * size
    O, lse = O.cpu().double(), lse.cpu().double()
    empty = rows[:, None] & (want_lse == -math.inf)
    seen = rows[:, None] & (want_lse != -math.inf)
    assert (O[empty] == 0).all() and (lse[empty] == -math.inf).all()
    bound = (2 ** -8 + 2 ** -12 + 2 * off) * weights + 2 ** -8 * want.abs() + 1e-30
    assert ((O - want).abs() <= bound)[seen].all(), float(((O - want).abs() / bound)[seen].max())
    assert ((lse - want_lse).abs()[seen] <= 2 ** -15 + 2 * off).all()


def sequences(c):
    return [(int(c.q_start[s]), c.q[s], c.first[s], c.k[s]) for s in range(c.S)]


def growing(c, steps):
    """Keys whose logits grow from step to step of 128, from each sequence's first on, by more than a row's reference (2^24 above the largest so far) leaves room
    for, and begin again: every third query the other way round, and every fourth alike in all steps."""
    for f, n in zip(c.first, c.k):
        for j in range(0, n, 128):
            c.K[f + j:f + min(j + 128, n)] = (torch.randn((min(128, n - j), c.Hkv, D), generator=torch.Generator().manual_seed(j)) * 0.1).to(torch.bfloat16)
            c.K[f + j:f + min(j + 128, n), :, 3] = float(steps[j // 128 % len(steps)])
    factor = torch.tensor([(1.0, -1.0, 0.0, 0.5)[i % 4] for i in range(c.T)])
    c.Q[:, :, 3] = (factor * 4.0)[:, None].to(torch.bfloat16)
    return c


# (steps 0, 60, 120 of dim 3: logits up to 4 x 120 / sqrt(128) = 42, 21 = 30 powers of two from step to step)
GROWING = {
    "rows": (ROWS16, dict(q=[16, 1, 9], k=[900, 400, 130], Hq=12, Hkv=12), dict(max_q=16)),
    "eight rows": (ROWS8, dict(q=[8, 1, 3], k=[900, 400, 130], Hq=4, Hkv=4), dict(max_q=8)),
    "tiles": (TILES, dict(q=[240, 200], k=[400, 1100], Hq=4, Hkv=2), {}),
    "shared tiles": (TILES, dict(q=[300], k=[4000], Hq=2, Hkv=2), {}),
    "pairs": (PAIRS, dict(q=[240, 600], k=[400, 1100], Hq=4, Hkv=2, pad_k=FAR), {}),
    "shared tiles of pairs": (PAIRS, dict(q=[300], k=[4000], Hq=2, Hkv=2, pad_k=FAR), {}),
    "pairs of three query heads": (PAIRS, dict(q=[500, 77], k=[3001, 640], Hq=6, Hkv=2, pad_k=FAR, layout="shuffled"), {}),
}


@pytest.mark.parametrize("name", GROWING)
def test_references_that_move(heart, kernel_of, name):
    kernel, kw, more = GROWING[name]
    for steps in ((0, 60, 120), (120, 60, 0), (60, 0, 120, 120)):
        c = growing(Case(**kw, seed=11, gain=0.5), steps)
        d = Device(heart, c, **more)
        assert kernel_of(d.cfg) == kernel
        O, lse = d.attention()
        assert heart.heart_get_status(d.ws) == 0
        near(c, sequences(c), torch.arange(c.T) < c.rows, O, lse)
        assert (O[c.rows:] == 77).all() and (lse[c.rows:] == 55).all()
        P, M = d.attention()
        assert same(O, P) and same(lse, M)


KINDS = {ROWS8: (dict(q=[3, 5], k=[50, 70], Hq=2), dict(max_q=4)), ROWS16: (dict(q=[16] * 8 + [4], k=[60, 9] * 4 + [70], Hq=8, Hkv=8), dict(max_q=16)),
         TILES: (dict(q=[400, 300], k=[50, 170], Hq=2), {}), PAIRS: (dict(q=[400, 300], k=[50, 170], Hq=2, Hkv=2, pad_k=FAR), {})}


@pytest.mark.parametrize("kernel", KINDS)
def test_states_that_are_not_finite(heart, kernel_of, kernel):
    """One of the last sequence's: its rows are not finite, the others as they are without it.  A logit of -inf has no weight."""
    kw, more = KINDS[kernel]
    last = len(kw["q"]) - 1
    first_row, rows = sum(kw["q"][:last]), sum(kw["q"])
    clean = Case(**kw)
    want, want_lse = Device(heart, clean, **more).attention()
    for what, where in ((math.nan, "K"), (math.inf, "V"), (-math.inf, "V"), (math.nan, "V")):
        c = Case(**kw)
        getattr(c, where)[c.first[last] + kw["k"][last] - 1, 0, 5] = what
        d = Device(heart, c, **more)
        assert kernel_of(d.cfg) == kernel
        O, lse = d.attention()
        assert same(O[:first_row], want[:first_row]) and same(lse[:first_row], want_lse[:first_row])
        heads = c.Hq // c.Hkv  # (those of key head 0)
        hit = O[first_row:rows, :heads].float()
        assert not torch.isfinite(hit).all(-1).any() and same(O[first_row:rows, heads:], want[first_row:rows, heads:])
        assert heart.heart_get_status(d.ws) == 0
    for at in (0, kw["k"][last] - 1):
        c = Case(**kw)
        c.Q[:, :, 5] = c.Q[:, :, 5].abs() + 1
        c.K[c.first[last] + at, :, 5] = -math.inf
        O, lse = Device(heart, c, **more).attention()
        of = sequences(c)
        r0, n, f, L = of[last]
        near_of = of[:last] + [(r0, n, f + 1, L - 1) if at == 0 else (r0, n, f, L - 1)]
        near(c, near_of, torch.arange(c.T) < rows, O, lse)


@pytest.mark.parametrize("kernel", KINDS)
def test_bad_arrays_touch_nothing_outside(heart, kernel_of, kernel):
    """Starts and lengths out of range are taken as the nearest valid ones: rows of one sequence are what these say, all around the tensors stays as it is."""
    kw, more = KINDS[kernel]
    GUARD = 300  # rows
    for what in ("starts", "far starts", "end", "far end", "descending", "length", "far length", "negative length", "first", "far first", "negative first"):
        c = Case(**kw, pad=0)
        big = (1 << 31) - 1
        if what in ("starts", "far starts"):
            c.q_start[0] = -2 if what == "starts" else -big - 1
        elif what in ("end", "far end"):
            c.q_start[c.S] = c.T + 1 if what == "end" else big
        elif what == "descending":
            c.q_start[1] = c.T + 2
        elif what in ("length", "far length", "negative length"):
            c.k_len[0] = {"length": c.Tk + 1, "far length": big, "negative length": -5}[what]
        else:
            c.k_start[0] = {"first": c.Tk - c.k[0] + 1, "far first": big, "negative first": -1}[what]
        d = Device(heart, c, **more)
        assert kernel_of(d.cfg) == kernel
        around_O = torch.full((c.T + 2 * GUARD, c.Hq, D), 77.0, dtype=torch.bfloat16, device="cuda")
        around_lse = torch.full((c.T + 2 * GUARD, c.Hq), 55.0, device="cuda")
        O, lse = around_O[GUARD:-GUARD], around_lse[GUARD:-GUARD]
        heart.heart_cross_attn(d.cfg, d.Q, d.K, d.V, *d.where, O, d.ws, lse=lse)
        assert heart.heart_get_status(d.ws) == heart.ERR_DEVICE_CHECK, what
        for x, as_it_was in ((around_O, 77), (around_lse, 55)):
            assert (x[:GUARD] == as_it_was).all() and (x[-GUARD:] == as_it_was).all(), what
        of, owners = [], torch.zeros(c.T, dtype=torch.int64)
        for s in range(c.S):
            r0 = min(max(int(c.q_start[s]), 0), c.T)
            r1 = min(max(int(c.q_start[s + 1]), r0), c.T)
            L = min(max(int(c.k_len[s]), 0), c.Tk)
            of.append((r0, r1 - r0, min(max(int(c.k_start[s]), 0), c.Tk - L), L))
            owners[r0:r1] += 1
        sure = owners == 1
        for r0, n, f, L in of:
            if not (torch.isfinite(c.K[f:f + L].float()).all() and torch.isfinite(c.V[f:f + L].float()).all()):
                sure[r0:r0 + n] = False  # (rows of no sequence, which hold no numbers)
        assert sure.any()
        near(c, [x for x in of if sure[x[0]:x[0] + x[1]].any()], sure, O, lse)
        none = owners == 0
        assert (O.cpu()[none] == 77).all() and (lse.cpu()[none] == 55).all()


LONG = [(ROWS16, dict(q=[4], k=[20000], Hq=64, Hkv=8, pad=0)), (TILES, dict(q=[370], k=[32761], Hq=1, Hkv=1)), (ROWS16, dict(q=[150], k=[9001], Hq=2, Hkv=2, layout="fused")),
        (ROWS16, dict(q=[30, 1, 0, 30], k=[14000, 77, 5, 16001], Hq=4, Hkv=2, layout="shuffled")), (PAIRS, dict(q=[260], k=[140000], Hq=1, Hkv=1))]


@pytest.mark.parametrize("case", range(len(LONG)))
def test_few_rows_over_long_states(heart, kernel_of, case):
    """Few tiles of many steps, which several CTAs share."""
    kernel, kw = LONG[case]
    c = Case(**kw, seed=case)
    d = Device(heart, c)
    assert kernel_of(d.cfg) == kernel
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    near(c, sequences(c), torch.arange(c.T) < c.rows, O, lse)
    P, M = d.attention()
    assert same(O, P) and same(lse, M)


@pytest.mark.parametrize("kernel,max_q,q,k", [(ROWS8, 1, [30000, 1, 0, 20000], [33, 1, 7, 0]), (ROWS16, 16, [20001, 16], [200, 33]), (ROWS8, 1, [1] * 40 + [30000], [20] * 41)])
def test_many_more_rows_than_max_q(heart, kernel_of, kernel, max_q, q, k):
    """The kernel for few rows with thousands of tiles of a sequence: right, if slow."""
    c = Case(q, k, Hq=2, Hkv=2, seed=max_q)
    d = Device(heart, c, max_q=max_q)
    assert kernel_of(d.cfg) == kernel
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    near(c, sequences(c), torch.arange(c.T) < c.rows, O, lse)
