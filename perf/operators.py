"""Operators on a paged cache of keys and values, as cases for timing.

A program that generates chunk by chunk (a few video frames at a time, or tokens) keeps the keys and values of the tokens
before in pages: `heart_cache_write` stores those of the new tokens, as bf16 or quantised to e4m3 with a power-of-two scale
for every token and head; `heart_cache_attn` is the attention of the new tokens over their sequences' pages;
`heart_cache_read` brings tokens back as bf16, for the calls that take whole tensors.

A case is a dict of plain values; `do` says which of the three it is.  Sequence s has kv_len[s] tokens in its pages, the
new ones included; the rows row_start[s] .. row_start[s + 1] of the packed tensors are its last ones.  Lengths come from the case
alone, all else from the seed.
"""
import math
import random

import torch

own = False

D = 128


def _case(name, do, kind, S, new, old, Hq, Hkv, page, causal=0, window=0, sink=0, lse=False, pad=0, head_major=False, lens=1):
    return {"name": name, "do": do, "kind": kind, "S": S, "new_lo": new[0], "new_hi": new[1], "old_lo": old[0], "old_hi": old[1],
            "Hq": Hq, "Hkv": Hkv, "page": page, "causal": causal, "window": window, "sink": sink, "lse": lse, "pad": pad,
            "head_major": head_major, "lens": lens}


def listed():
    return [
        # One decoding step of a small batch: the new token's keys and values, quantised; launch latency.
        _case("write_tokens_8x8_e4m3", "write", "e4m3", 8, (1, 1), (100, 2000), 8, 8, 64),
        # Prompts of several users in one packed batch, padded to the size of a captured graph.
        _case("write_prompts_5x12_bf16", "write", "bf16", 5, (1, 900), (0, 700), 12, 12, 16, pad=37),
        # Three latent frames of Wan2.1-14B at 480P with guidance (two sequences), quantised as they are written.
        _case("write_frames_2x40_e4m3", "write", "e4m3", 2, (4680, 4680), (0, 0), 40, 40, 128),
        # Moving a few short contexts out of their pages.
        _case("read_short_3x4_e4m3", "read", "e4m3", 3, (1, 500), (0, 0), 4, 4, 16),
        # Contexts of a batch, the last tokens of each.
        _case("read_batch_16x8_bf16", "read", "bf16", 16, (1, 4000), (0, 900), 8, 8, 64),
        # A whole 480P context of Wan2.1-14B as the [H, N, D] tensors that a sparse layer-step takes.
        _case("read_context_40x33k_e4m3", "read", "e4m3", 1, (32760, 32760), (0, 0), 40, 40, 128, head_major=True),
        # One token of one sequence, shared heads: latency.
        _case("attend_token_1x32_4k_bf16", "attend", "bf16", 1, (1, 1), (4099, 4099), 32, 8, 64),
        # A decoding batch over contexts of very different lengths, quantised cache.
        _case("attend_tokens_64x32_16k_e4m3", "attend", "e4m3", 64, (1, 1), (200, 16000), 32, 8, 64, causal=1, lens=3),
        # A decoding batch of a model without shared heads.
        _case("attend_tokens_16x12_8k_bf16", "attend", "bf16", 16, (1, 1), (500, 8000), 12, 12, 32, lens=2),
        # Prompts and single tokens mixed, token-causal, a window with sink tokens, three queries a head, small pages, log-sum-exp.
        _case("attend_prompts_6x24_bf16", "attend", "bf16", 6, (1, 1500), (0, 3000), 24, 8, 16, causal=1, window=2048, sink=4, lse=True,
              pad=21),
        # Three frames of Wan2.1-1.3B at 480P over their context, causal by frames.
        _case("attend_frames_12x33k_bf16", "attend", "bf16", 1, (4680, 4680), (28080, 28080), 12, 12, 64, causal=1560, lse=True),
        # Three frames of Wan2.1-14B at 480P over a quantised context, every query sees all of it.
        _case("attend_frames_40x33k_e4m3", "attend", "e4m3", 1, (4680, 4680), (28080, 28080), 40, 40, 128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    do = rng.choice(["write", "read", "attend", "attend", "attend", "attend"])
    kind = rng.choice(["bf16", "e4m3"])
    page = rng.choice([16, 32, 64, 128])
    Hkv = rng.choice([1, 2, 4, 5, 8, 12, 24, 40])
    if do != "attend":
        S = _log_int(rng, 1, 64)
        hi = max(1, min(32760, 32760 * 40 // (S * Hkv)))
        new = _log_int(rng, 1, hi)
        old = rng.choice([0, _log_int(rng, 1, hi)])
        return {"do": do, "kind": kind, "S": S, "new_lo": max(1, new // rng.choice([1, 4])), "new_hi": new, "old_lo": 0, "old_hi": old,
                "Hq": Hkv, "Hkv": Hkv, "page": page, "causal": 0, "window": 0, "sink": 0, "lse": False,
                "pad": rng.choice([0, 0, rng.randint(1, 50)]), "head_major": rng.random() < 0.3, "lens": rng.randint(1, 1 << 20)}
    G = rng.choice([1, 1, 2, 3, 4, 8])
    while G * Hkv > 64:
        G = max(1, G // 2)
    if rng.random() < 0.5:  # tokens, or a few drafted ones, of a batch
        S, new_hi = _log_int(rng, 1, 64), rng.choice([1, 1, 1, rng.randint(2, 9)])
        old_hi = _log_int(rng, 1, 16000)
        new_lo, old_lo = 1, max(0, old_hi // rng.choice([1, 3, 80]))
    else:  # prompts and frames
        S, new_hi = _log_int(rng, 1, 8), _log_int(rng, 10, 4680)
        old_hi = rng.choice([0, _log_int(rng, 10, 28080)])
        new_lo, old_lo = max(1, new_hi // rng.choice([1, 4, 50])), old_hi // rng.choice([1, 2])
    # what a plain computation holds in memory is bounded: the padded scores, the gathered keys and values
    while S > 1 and (S * new_hi * (new_hi + old_hi) * G * Hkv > 4680 * 32760 * 40 or S * (new_hi + old_hi) * Hkv * (4 if kind == "bf16" else 2) > 1.1e9 / D):
        S = max(1, S // 2)
    causal = rng.choice([0, 1, 1, rng.randint(2, 1560)])
    window = rng.choice([0, 0, _log_int(rng, 1, 8000)])
    return {"do": do, "kind": kind, "S": S, "new_lo": new_lo, "new_hi": new_hi, "old_lo": old_lo, "old_hi": old_hi, "Hq": G * Hkv,
            "Hkv": Hkv, "page": page, "causal": causal, "window": window, "sink": rng.choice([0, rng.randint(1, 200)]) if window else 0,
            "lse": rng.random() < 0.5, "pad": rng.choice([0, 0, rng.randint(1, 50)]), "head_major": False, "lens": rng.randint(1, 1 << 20)}


def _lengths(c):
    """New tokens and context length of every sequence."""
    rng = random.Random(c["lens"])
    new = [rng.randint(c["new_lo"], c["new_hi"]) for _ in range(c["S"])]
    return new, [n + rng.randint(c["old_lo"], c["old_hi"]) for n in new]


def _visible(c, n, L):
    """(pairs of a query and a key that it sees, keys that some query sees) of a sequence."""
    pairs, keys = 0, 0
    g, w = c["causal"], c["window"]
    seen_to, sink = 0, 0  # keys are counted in order: windows only move up
    step = 1 if g else n
    for p in range(L - n, L, step):
        end = min(L, (p // g + 1) * g) if g else L
        lo = max(0, end - w) if w else 0
        low = min(c["sink"], lo)
        pairs += (end - lo + low) * (1 if g else n)
        sink = max(sink, low)
        keys += end - max(lo, seen_to)
        seen_to = end
        first = lo if p == L - n else first
    return pairs, keys + min(sink, first)


def work(c):
    """Every new row and every key that is seen read once, results written once; two products for each visible pair."""
    new, lens = _lengths(c)
    element = 2 if c["kind"] == "bf16" else 1 + 1 / D  # (a byte of scale for 128 elements)
    if c["do"] != "attend":
        rows = sum(new) * c["Hkv"]
        return {"bytes": 2 * rows * D * (2 + element), "flops": 2 * rows * D * (c["kind"] == "e4m3")}
    seen = [_visible(c, n, L) for n, L in zip(new, lens)]
    return {"bytes": sum(new) * c["Hq"] * (D * 4 + 4 * c["lse"]) + 2 * D * element * c["Hkv"] * sum(k for _, k in seen),
            "flops": 4 * D * c["Hq"] * sum(p for p, _ in seen)}


# ---------------------------------------------------------------- inputs


def prepare(c, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    new, lens = _lengths(c)
    S, Hq, Hkv, page, e4m3 = c["S"], c["Hq"], c["Hkv"], c["page"], c["kind"] == "e4m3"

    def normal(*shape, gain=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * gain).to(torch.bfloat16)

    pages = [-(-n // page) for n in lens]
    n_pages = sum(pages) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    width = max(pages)
    first = torch.tensor([sum(pages[:s]) for s in range(S)], device="cuda")
    index = first[:, None] + torch.arange(width, device="cuda")
    table = torch.where(torch.arange(width, device="cuda") < torch.tensor(pages, device="cuda")[:, None],
                        order[index.clamp(max=n_pages - 1)], torch.zeros_like(order[:1]))
    s = {"c": c, "T": sum(new) + c["pad"], "n": sum(new), "n_max": max(new), "L_max": max(lens), "table": table.contiguous(),
         "row_start": torch.tensor([sum(new[:i]) for i in range(S + 1)], dtype=torch.int32, device="cuda"),
         "kv_len": torch.tensor(lens, dtype=torch.int32, device="cuda"), "lens": lens, "new": new, "n_pages": n_pages}
    # the pools as earlier calls left them; keys with channels of different strength, as projections give them
    gain = torch.rand((Hkv, 1, D), generator=gen, device="cuda") * 1.2 + 0.3
    for x in ("k", "v"):
        pool = normal(n_pages, Hkv, page, D, gain=gain if x == "k" else 1.0)
        s[x], s[x + "_scale"] = _quantise(pool) if e4m3 else (pool, None)
    if c["do"] == "write":
        s["K"], s["V"] = normal(s["T"], Hkv, D, gain=gain[:, 0]), normal(s["T"], Hkv, D)
    elif c["do"] == "read":
        for x in ("K", "V"):
            s[x] = normal(*((Hkv, s["T"], D) if c["head_major"] else (s["T"], Hkv, D)))
    else:
        s["Q"], s["O"] = normal(s["T"], Hq, D, gain=1.3), normal(s["T"], Hq, D)
        s["lse"] = torch.zeros((s["T"], Hq), device="cuda") if c["lse"] else None
    if own:
        s["config"], s["cache"], s["workspace"] = _handles(s)
    return s


def _handles(s):
    """What a program keeps from call to call: the shapes, the cache's handle, a workspace."""
    from paper_2605_14513_b200 import heart

    c = s["c"]
    cfg = heart.make_cache_config(c["S"], s["T"], c["Hq"], c["Hkv"], c["page"], s["n_pages"], s["table"].shape[1],
                                  kind=heart.CACHE_E4M3 if c["kind"] == "e4m3" else heart.CACHE_BF16, max_new=s["n_max"],
                                  causal=c["causal"], window=c["window"], sink=c["sink"],
                                  kv_strides=(D, s["T"] * D) if c["do"] == "read" and c["head_major"] else (0, 0))
    return cfg, heart.Cache(cfg, s["k"], s["v"], s["k_scale"], s["v_scale"]), heart.new_cache_workspace(cfg)


# ---------------------------------------------------------------- plain forms


def _quantise(x):
    """e4m3 codes and scale bytes: the scale is the smallest power of two (from 2^-110) under which no magnitude exceeds 448."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m > 0, e - 9 + (m > 0.875).int(), -110).clamp(min=-110)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _bytes(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _rows(s):
    """Sequence, place among its new tokens and position of every row that belongs to a sequence."""
    row = torch.arange(s["n"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["row_start"], row, right=True) - 1
    place = row - s["row_start"][seq]
    return seq, place, s["kv_len"][seq] - (s["row_start"][seq + 1] - row)


def _tokens(s, x, seq, pos):
    """Tokens out of a pool, in 32 bits: [.., Hkv, D] for tensors of sequences and positions."""
    page, slot = s["table"][seq, pos // s["c"]["page"]].long(), (pos % s["c"]["page"]).long()
    got = _bytes(s[x])[page, :, slot]
    if s[x + "_scale"] is None:
        return got.float()
    return got.view(torch.float8_e4m3fn).float() * torch.exp2(s[x + "_scale"][page, :, slot].float() - 127)[..., None]


def _plain_write(s):
    seq, _, pos = _rows(s)
    page, slot = s["table"][seq, pos // s["c"]["page"]].long(), (pos % s["c"]["page"]).long()
    if s["k_scale"] is None:
        s["k"][page, :, slot], s["v"][page, :, slot] = s["K"][:s["n"]], s["V"][:s["n"]]
        return
    k, k_scale = _quantise(s["K"][:s["n"]])
    v, v_scale = _quantise(s["V"][:s["n"]])
    _bytes(s["k"])[page, :, slot], _bytes(s["v"])[page, :, slot] = _bytes(k), _bytes(v)
    s["k_scale"][page, :, slot], s["v_scale"][page, :, slot] = k_scale, v_scale


def _plain_read(s):
    seq, _, pos = _rows(s)
    K, V = _tokens(s, "k", seq, pos).to(torch.bfloat16), _tokens(s, "v", seq, pos).to(torch.bfloat16)
    if s["c"]["head_major"]:
        s["K"][:, :s["n"]], s["V"][:, :s["n"]] = K.transpose(0, 1), V.transpose(0, 1)
    else:
        s["K"][:s["n"]], s["V"][:s["n"]] = K, V


def _plain_attend(s):
    """All sequences at once, padded to the longest."""
    c = s["c"]
    S, Hq, Hkv, n, L = c["S"], c["Hq"], c["Hkv"], s["n_max"], s["L_max"]
    lens, new = s["kv_len"][:, None], s["row_start"].diff()[:, None]
    every = torch.arange(L, device="cuda", dtype=torch.int32)[None]
    seq = torch.arange(S, device="cuda")[:, None]
    row = torch.arange(n, device="cuda", dtype=torch.int32)[None]
    q = s["Q"][(s["row_start"][:-1, None] + row).clamp(max=s["T"] - 1).long()].float()
    q = q.view(S, n, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, D)
    held = every.minimum(lens - 1)  # (places behind a sequence's end take its last token; they are masked)
    p = (q * D ** -0.5) @ _tokens(s, "k", seq, held).permute(0, 2, 3, 1)
    pos = lens - new + row
    end = lens.expand(-1, n) if c["causal"] == 0 else lens.minimum((torch.div(pos, c["causal"], rounding_mode="floor") + 1) * c["causal"])
    low = end - c["window"] if c["window"] else torch.zeros_like(end)
    hidden = (every[:, None] >= end[..., None]) | ((every[:, None] < low[..., None]) & (every[:, None] >= c["sink"]))
    p.view(S, Hkv, n, Hq // Hkv, L).masked_fill_(hidden[:, None, :, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ _tokens(s, "v", seq, held).transpose(1, 2)) / total
    seq, place, _ = _rows(s)
    s["O"][:s["n"]] = o.view(S, Hkv, n, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(S, n, Hq, D)[seq, place].to(torch.bfloat16)
    if s["lse"] is not None:
        lse = (top + total.log()).view(S, Hkv, n, Hq // Hkv).permute(0, 2, 1, 3).reshape(S, n, Hq)
        s["lse"][:s["n"]] = lse[seq, place]


def _own(s):
    from paper_2605_14513_b200 import heart

    where = s["table"], s["row_start"], s["kv_len"]
    if s["c"]["do"] == "write":
        heart.heart_cache_write(s["config"], s["K"], s["V"], s["cache"], *where, s["workspace"])
    elif s["c"]["do"] == "read":
        heart.heart_cache_read(s["config"], s["cache"], *where, s["K"], s["V"], s["workspace"])
    else:
        heart.heart_cache_attn(s["config"], s["Q"], s["cache"], *where, s["O"], s["workspace"], lse=s["lse"])


def run(s):
    if own:
        _own(s)
    else:
        {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[s["c"]["do"]](s)
    if s["c"]["do"] == "write":
        return {x: s[x] for x in ("k", "v", "k_scale", "v_scale") if s[x] is not None}
    if s["c"]["do"] == "read":
        return {"K": s["K"], "V": s["V"]}
    return {"O": s["O"]} if s["lse"] is None else {"O": s["O"], "lse": s["lse"]}


# ---------------------------------------------------------------- the definition in 64 bits


def exact(c, seed):
    s = prepare(c, seed)
    page = c["page"]
    value = {x: s[x].to(torch.float32).double() for x in ("k", "v")}
    weight = {x: None if s[x + "_scale"] is None else torch.pow(2.0, s[x + "_scale"].double() - 127) for x in ("k", "v")}
    starts = [sum(s["new"][:i]) for i in range(c["S"])]

    def where(i, lo, hi):  # pages and slots of tokens lo .. hi - 1 of sequence i
        pos = torch.arange(lo, hi, device="cuda")
        return s["table"][i].long()[pos // page], pos % page

    if c["do"] == "write":
        out = dict(value)
        for i in range(c["S"]):
            pg, slot = where(i, s["lens"][i] - s["new"][i], s["lens"][i])
            for x, given in (("k", "K"), ("v", "V")):
                rows = s[given][starts[i]:starts[i] + s["new"][i]].double()
                if c["kind"] == "bf16":
                    out[x][pg, :, slot] = rows
                    continue
                m, e = torch.frexp(rows.abs().amax(-1) / 448)
                e = torch.where(m > 0, e - (m == 0.5).int(), -110).clamp(min=-110)
                rows = torch.ldexp(rows, -e[..., None])
                # four significant bits, steps of 2^-9 at the low end; rounding to even
                unit = torch.ldexp(torch.ones_like(rows), (torch.frexp(rows)[1] - 4).clamp(min=-9))
                out[x][pg, :, slot] = torch.round(rows / unit) * unit
        return {x: out[x] if x in out else None for x in (("k", "v") if c["kind"] == "bf16" else ("k", "v", "k_scale", "v_scale"))}
    if c["do"] == "read":
        out = {x: s[x].double() for x in ("K", "V")}
        for i in range(c["S"]):
            pg, slot = where(i, s["lens"][i] - s["new"][i], s["lens"][i])
            for x, to in (("k", "K"), ("v", "V")):
                rows = value[x][pg, :, slot]
                if weight[x] is not None:
                    rows = rows * weight[x][pg, :, slot][..., None]
                if c["head_major"]:
                    out[to][:, starts[i]:starts[i] + s["new"][i]] = rows.transpose(0, 1)
                else:
                    out[to][starts[i]:starts[i] + s["new"][i]] = rows
        return out
    O, G = s["O"].double(), c["Hq"] // c["Hkv"]
    lse = None if s["lse"] is None else s["lse"].double()
    for i in range(c["S"]):
        n, L = s["new"][i], s["lens"][i]
        pg, slot = where(i, 0, L)
        pos = torch.arange(L - n, L, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None]
        seen = torch.ones((n, L), dtype=torch.bool, device="cuda")
        end = torch.full_like(pos, L)
        if c["causal"]:
            end = torch.minimum(end, (pos // c["causal"] + 1) * c["causal"])
            seen &= j < end
        if c["window"]:
            seen &= (j >= end - c["window"]) | (j < c["sink"])
        for h in range(c["Hkv"]):
            k, v = value["k"][pg, h, slot], value["v"][pg, h, slot]
            if weight["k"] is not None:
                k, v = k * weight["k"][pg, h, slot][:, None], v * weight["v"][pg, h, slot][:, None]
            for g in range(h * G, h * G + G):
                logits = torch.where(seen, s["Q"][starts[i]:starts[i] + n, g].double() @ k.T / math.sqrt(D), -math.inf)
                total = torch.logsumexp(logits, -1, keepdim=True)
                O[starts[i]:starts[i] + n, g] = torch.exp(logits - total) @ v
                if lse is not None:
                    lse[starts[i]:starts[i] + n, g] = total[:, 0]
    return {"O": O} if lse is None else {"O": O, "lse": lse}
