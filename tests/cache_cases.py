"""Small paged caches for the tests: inputs, the definition in 64 bits, and the calls."""
import math

import numpy as np
import torch

D = 128


def quantise(x):
    """Codes and scale bytes by the definition, in 64 bits on the CPU; rows that are not finite: codes 0, byte 255."""
    x = x.double()
    top = x.abs().amax(-1)
    fine = torch.isfinite(top)
    m, e = torch.frexp(torch.where(fine, top, torch.ones_like(top)) / 448)
    e = torch.where(m == 0, torch.full_like(e, -110), e - (m == 0.5).int()).clamp(min=-110)
    x = torch.where(fine[..., None], x, torch.zeros_like(x)).clamp(-1.875 * 2.0 ** 127, 1.875 * 2.0 ** 127)
    y = torch.ldexp(x, -e[..., None])
    unit = torch.ldexp(torch.ones_like(y), (torch.frexp(y)[1] - 4).clamp(min=-9))  # four bits, steps of 2^-9 at least
    codes = (torch.round(y / unit) * unit).to(torch.float8_e4m3fn)
    return codes, torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)


def dequantise(codes, scale):
    w = torch.where(scale == 255, torch.full_like(scale, 1, dtype=torch.float64) * math.nan, torch.exp2(scale.double() - 127))
    return codes.double() * w[..., None]


class Case:
    """lens, new: tokens and new tokens of each sequence.  All tensors on the CPU; `on(device)` brings them over."""

    def __init__(self, lens, new, Hq=2, Hkv=1, page=16, kind="bf16", causal=0, window=0, sink=0, scale=0.0, pad=3, seed=0, garbage=True,
                 layout="head", gain=1.3, spare=2):
        self.lens, self.new, self.Hq, self.Hkv, self.page, self.kind = list(lens), list(new), Hq, Hkv, page, kind
        self.causal, self.window, self.sink, self.scale = causal, window, sink, scale
        g = torch.Generator().manual_seed(seed)
        S = len(self.lens)
        self.S, self.T = S, sum(self.new) + pad
        pages = [-(-n // page) for n in self.lens]
        self.n_pages = sum(pages) + spare
        self.width = max(max(pages), 1)
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((S, self.width), -7, dtype=torch.int32)  # (entries of no token are not looked at)
        for s in range(S):
            self.table[s, :pages[s]] = order[sum(pages[:s]):sum(pages[:s + 1])]
        self.row_start = torch.tensor([sum(self.new[:s]) for s in range(S + 1)], dtype=torch.int32)
        self.kv_len = torch.tensor(self.lens, dtype=torch.int32)

        def normal(*shape, k=1.0):
            return (torch.randn(shape, generator=g) * k).to(torch.bfloat16)

        self.Q = normal(self.T, Hq, D, k=gain)
        self.K, self.V = normal(self.T, Hkv, D), normal(self.T, Hkv, D)
        pool = [normal(self.n_pages, Hkv, page, D) for _ in range(2)]
        if garbage:  # behind the sequences' ends, and in pages of no sequence
            used = torch.zeros((self.n_pages, page), dtype=torch.bool)
            for s in range(S):
                j = torch.arange(self.lens[s])
                used[self.table[s].long()[j // page], j % page] = True
            for x in pool:
                x[~used[:, None, :].expand(-1, Hkv, -1)] = torch.tensor([math.nan, math.inf, -math.inf, 1e30] * 32, dtype=torch.bfloat16)
        self.k_scale = self.v_scale = None
        if kind == "e4m3":
            (self.k, self.k_scale), (self.v, self.v_scale) = (quantise(x) for x in pool)
        else:
            self.k, self.v = pool
        self.layout = layout
        if layout == "token":  # [n_pages, page, Hkv, D] in memory
            self.k, self.v = (self._as(x) for x in (self.k, self.v))

    @staticmethod
    def _as(x):
        return _bytes(x).transpose(1, 2).contiguous().transpose(1, 2).view(x.dtype) if x.element_size() == 1 else x.transpose(1, 2).contiguous().transpose(1, 2)

    def config(self, heart, **kw):
        kw.setdefault("max_new", max(self.new))
        if self.layout == "token":
            kw["pool_strides"] = (self.page * self.Hkv * D, D, self.Hkv * D)
        return heart.make_cache_config(self.S, self.T, self.Hq, self.Hkv, self.page, self.n_pages, self.width,
                                       kind=heart.CACHE_E4M3 if self.kind == "e4m3" else heart.CACHE_BF16, causal=self.causal,
                                       window=self.window, sink=self.sink, scale=self.scale, **kw)

    def values(self):
        """Keys and values of the pools in 64 bits."""
        if self.kind == "e4m3":
            return dequantise(self.k, self.k_scale), dequantise(self.v, self.v_scale)
        return self.k.double(), self.v.double()

    def tokens(self, pool, s):
        j = torch.arange(self.lens[s])
        return pool[self.table[s].long()[j // self.page], :, j % self.page]  # [len, Hkv, D]

    def seen(self, s):
        """[new, len]: which tokens each new token sees."""
        n, L = self.new[s], self.lens[s]
        p = torch.arange(L - n, L)[:, None]
        j = torch.arange(L)[None]
        end = torch.full_like(p, L) if self.causal == 0 else torch.clamp((p // self.causal + 1) * self.causal, max=L)
        ok = (j < end) & (p >= 0)
        if self.window:
            ok &= (j >= end - self.window) | (j < self.sink)
        return ok

    def attention(self):
        """O and lse of the rows that belong to a sequence, fp64 [T, Hq, D] and [T, Hq]; other rows NaN."""
        k, v = self.values()
        O = torch.full((self.T, self.Hq, D), math.nan, dtype=torch.float64)
        lse = torch.full((self.T, self.Hq), math.nan, dtype=torch.float64)
        scale = self.scale if self.scale > 0 else 1 / math.sqrt(D)
        G = self.Hq // self.Hkv
        for s in range(self.S):
            r0, n = int(self.row_start[s]), self.new[s]
            ks, vs, ok = self.tokens(k, s), self.tokens(v, s), self.seen(s)
            for h in range(self.Hq):
                logits = self.Q[r0:r0 + n, h].double() @ ks[:, h // G].T * scale
                logits = torch.where(ok, logits, torch.full_like(logits, -math.inf))
                total = torch.logsumexp(logits, -1) if self.lens[s] else torch.full((n,), -math.inf, dtype=torch.float64)
                w = torch.where(ok, torch.exp(logits - torch.where(total == -math.inf, torch.zeros_like(total), total)[:, None]), torch.zeros_like(logits))
                O[r0:r0 + n, h] = torch.where(ok.T[:, :, None], w.T[:, :, None] * vs[:, h // G][:, None], 0.0).sum(0) if n * self.lens[s] < 40000 else w @ vs[:, h // G]
                lse[r0:r0 + n, h] = total
        return O, lse

    def weight_bound(self):
        """sum_j w_j |v_j| for each row, as attention(): what roundings of the weights are relative to."""
        k, v = self.values()
        B = torch.zeros((self.T, self.Hq, D), dtype=torch.float64)
        scale = self.scale if self.scale > 0 else 1 / math.sqrt(D)
        G = self.Hq // self.Hkv
        for s in range(self.S):
            r0, n = int(self.row_start[s]), self.new[s]
            ks, vs, ok = self.tokens(k, s), self.tokens(v, s), self.seen(s)
            if not self.lens[s]:
                continue
            for h in range(self.Hq):
                logits = torch.where(ok, self.Q[r0:r0 + n, h].double() @ ks[:, h // G].T * scale, torch.tensor(-math.inf, dtype=torch.float64))
                w = torch.nan_to_num(torch.softmax(logits, -1), 0.0)
                B[r0:r0 + n, h] = w @ vs[:, h // G].abs()
        return B


def _bytes(x):
    return x.view(torch.uint8)


class Device:
    """The case's tensors on a GPU and the library's handles."""

    def __init__(self, heart, c, device="cuda", **kw):
        self.c, self.heart = c, heart
        self.cfg = c.config(heart, **kw)

        def up(x):
            if x is None:
                return None
            y = x.view(torch.uint8).to(device).view(x.dtype) if x.dtype == torch.float8_e4m3fn else x.to(device)
            return y if y.stride() == x.stride() else torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=device).copy_(y)

        self.cache = heart.Cache(self.cfg, up(c.k), up(c.v), up(c.k_scale), up(c.v_scale))
        self.where = up(c.table), up(c.row_start), up(c.kv_len)
        self.Q, self.K, self.V = up(c.Q), up(c.K), up(c.V)
        self.ws = heart.new_cache_workspace(self.cfg, device=device)

    def attention(self, lse=True):
        O = torch.full_like(self.Q, 77.0)
        L = torch.full((self.c.T, self.c.Hq), 55.0, device=self.Q.device) if lse else None
        self.heart.heart_cache_attn(self.cfg, self.Q, self.cache, *self.where, O, self.ws, lse=L)
        return O, L


def check_attention(c, O, lse, status=0):
    """Against the definition.  Rows of no sequence are as they were (77, 55)."""
    want, want_lse = c.attention()
    n = int(c.row_start[-1])
    O, lse = O.cpu(), lse.cpu()
    assert (O[n:] == 77).all() and (lse[n:] == 55).all()
    got, got_lse = O[:n].double(), lse[:n].double()
    want, want_lse = want[:n], want_lse[:n]
    empty = want_lse == -math.inf
    assert (got[empty] == 0).all() and (got_lse[empty] == -math.inf).all()
    # A weight is rounded to bf16 once (half a step: 2^-8 of it), the result once more; products are exact in 32 bits, their sums
    # off by less than 2^-17 of the sum of magnitudes (128 to some 10^4 terms, each sum rounded by 2^-24; the exponent's argument, up to
    # 2^6, by 2^-18 of one: weights by as much).
    bound = (2 ** -8 + 2 ** -12) * c.weight_bound()[:n] + 2 ** -8 * want.abs() + 1e-30
    worst = ((got - want).abs() / bound)[~empty]
    assert worst.numel() == 0 or worst.max() <= 1.0, float(worst.max())
    off = (got_lse - want_lse)[~empty].abs()
    assert off.numel() == 0 or off.max() <= 2 ** -14, float(off.max())  # (logits up to 2^6, 32-bit sums of 128 products)
    return got, want
