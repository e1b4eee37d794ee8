"""Cross attention, and the page tables of a cache built on the GPU, as cases for timing.

A layer of a video model, or of a decoder with an encoder, has the tokens of its sequences attend to states of another
length (a prompt's, a reference's): `heart_cross_attn`, packed rows of queries over packed or padded rows of keys and values.
A program that serves requests over a paged cache keeps a list of free pages; before every step `heart_cache_extend` gives the
sequences the pages that their new tokens need and writes what the calls on the cache read (page table, row starts, lengths) and
every row's slot, and behind it `heart_cache_release` takes back the pages of the requests that have ended.

A case is a dict of plain values; `do` says which of the three it is.  Lengths come from the case alone, all else from the seed.
"""
import math
import random

import torch

own = False

D = 128


def _cross(name, S, q, k, Hq, Hkv, lse=False, pad=0, layout="packed", lens=1):
    """Sequences of q[0] .. q[1] tokens over k[0] .. k[1] states.  layout: "packed" states one sequence behind the other, "padded" ones all of
    them k[1] rows apart, or "fused": packed, with keys and values as the two halves of one projection's rows."""
    return {"name": name, "do": "cross", "S": S, "q_lo": q[0], "q_hi": q[1], "k_lo": k[0], "k_hi": k[1], "Hq": Hq, "Hkv": Hkv, "lse": lse,
            "pad": pad, "layout": layout, "lens": lens}


def _extend(name, S, new, old, page, pad=0, slots=True, lens=1):
    return {"name": name, "do": "extend", "S": S, "new_lo": new[0], "new_hi": new[1], "old_lo": old[0], "old_hi": old[1], "page": page,
            "pad": pad, "slots": slots, "lens": lens}


def _release(name, S, old, page, ended, lens=1):
    return {"name": name, "do": "release", "S": S, "old_lo": old[0], "old_hi": old[1], "page": page, "ended": ended, "lens": lens}


def listed():
    return [
        # One token of one sequence over an encoder's states, shared heads: latency.
        _cross("cross_token_1x32_1500", 1, (1, 1), (1500, 1500), 32, 8),
        # A decoding batch over states of very different lengths, keys and values from one projection.
        _cross("cross_tokens_64x12_4k", 64, (1, 1), (100, 4000), 12, 12, layout="fused", lens=3),
        # Prompts and single tokens of several users over short states, one of them without any, three queries a head, log-sum-exp, rows behind
        # the last sequence (a captured graph's size).
        _cross("cross_prompts_6x24_512", 6, (1, 1500), (0, 512), 24, 8, lse=True, pad=21, lens=9),
        # Three latent frames of Wan2.1-1.3B at 480P over a text of 512 tokens.
        _cross("cross_chunk_1x12_4680x512", 1, (4680, 4680), (512, 512), 12, 12),
        # Whole sequences of Wan2.1-14B at 480P with guidance: two texts, padded to 512.
        _cross("cross_frames_2x40_33kx512", 2, (32760, 32760), (230, 512), 40, 40, layout="padded", lens=2),
        # A thousand tokens over a reference as long as a 480P sequence: few tiles, many keys.
        _cross("cross_reference_1x12_1000x33k", 1, (1000, 1000), (32760, 32760), 12, 12, lse=True),
        # One decoding step of a small batch.
        _extend("extend_tokens_64", 64, (1, 1), (1, 4000), 64),
        # Prompts of several users, some of them with cached tokens, rows behind the last sequence.
        _extend("extend_prompts_8x4k", 8, (1, 4680), (0, 3000), 16, pad=37),
        # A large batch in small pages, prompts and tokens mixed.
        _extend("extend_batch_1024x1k", 1024, (0, 1000), (0, 2000), 16),
        # A few requests of a batch have ended.
        _release("release_some_64", 64, (1, 4000), 64, 0.2),
        # Half of a large batch has ended, long contexts in small pages.
        _release("release_half_1024x16k", 1024, (0, 16000), 16, 0.5),
    ]


MOST_PAIRS = 2 * 40 * 32760 * 512  # of queries and states, over all heads
MOST_ROWS = 2 * 40 * 32760         # of queries, over all heads
MOST_STATES = 12 * 32760 * 2       # of keys, over all heads
MOST_SLOTS = 500_000


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    do = rng.choice(["cross", "cross", "cross", "extend", "release"])
    seed = rng.randint(1, 1 << 20)
    if do == "cross":
        Hkv = rng.choice([1, 2, 4, 5, 8, 12, 24, 40])
        G = rng.choice([1, 1, 2, 3, 4, 8])
        while G * Hkv > 64:
            G = max(1, G // 2)
        if rng.random() < 0.4:  # tokens, or a few drafted ones, of a batch
            S, q_hi = _log_int(rng, 1, 64), rng.choice([1, 1, 1, rng.randint(2, 9)])
            q_lo, k_hi = 1, _log_int(rng, 1, 8000)
        else:
            S, q_hi = _log_int(rng, 1, 8), _log_int(rng, 10, 32760)
            q_lo, k_hi = max(1, q_hi // rng.choice([1, 4, 50])), rng.choice([_log_int(rng, 1, 1500), _log_int(rng, 1, 32760)])
        while S > 1 and (S * q_hi * k_hi * G * Hkv > MOST_PAIRS or S * q_hi * G * Hkv > MOST_ROWS or S * k_hi * Hkv > MOST_STATES):
            S = max(1, S // 2)
        q_hi = max(1, min(q_hi, MOST_ROWS // (S * G * Hkv), MOST_PAIRS // (S * k_hi * G * Hkv)))
        k_hi = max(1, min(k_hi, MOST_STATES // (S * Hkv)))
        c = _cross("", S, (min(q_lo, q_hi), q_hi), (k_hi // rng.choice([1, 1, 3, 80]), k_hi), G * Hkv, Hkv, rng.random() < 0.5,
                   rng.choice([0, 0, rng.randint(1, 50)]), rng.choice(["packed", "padded", "fused"]), seed)
    elif do == "extend":
        S = _log_int(rng, 1, 1024)
        new = rng.choice([1, _log_int(rng, 1, min(4680, 2 * MOST_SLOTS // S))])
        old = rng.choice([0, _log_int(rng, 1, 16000)])
        c = _extend("", S, (rng.choice([0, new // 4, new]), new), (0, old), rng.choice([16, 32, 64, 128]), rng.choice([0, 0, rng.randint(1, 50)]),
                    rng.random() < 0.7, seed)
    else:
        S = _log_int(rng, 1, 1024)
        old = _log_int(rng, 1, 16000)
        c = _release("", S, (rng.choice([0, old // 4, old]), old), rng.choice([16, 32, 64, 128]), rng.choice([0.1, 0.5, 1.0]), seed)
    del c["name"]
    return c


def _lengths(c):
    """cross: tokens and states of every sequence; extend: new and old tokens; release: old ones, and which sequences have ended."""
    rng = random.Random(c["lens"])
    S = c["S"]
    if c["do"] == "cross":
        q = [rng.randint(c["q_lo"], c["q_hi"]) for _ in range(S)]
        k = [rng.randint(c["k_lo"], c["k_hi"]) for _ in range(S)]
        if c["k_lo"] == 0 and S > 1:
            k[rng.randrange(S)] = 0
        return q, k
    if c["do"] == "extend":
        return [rng.randint(c["new_lo"], c["new_hi"]) for _ in range(S)], [rng.randint(c["old_lo"], c["old_hi"]) for _ in range(S)]
    return [rng.randint(c["old_lo"], c["old_hi"]) for _ in range(S)], [rng.random() < c["ended"] for _ in range(S)]


def work(c):
    """cross: rows of queries and states read once, results written once, two products for each pair of them.  extend, release: lengths, list and
    table entries and slots that are read or written, once."""
    a, b = _lengths(c)
    if c["do"] == "cross":
        return {"bytes": sum(a) * c["Hq"] * (4 * D + 4 * c["lse"]) + 4 * D * c["Hkv"] * sum(b),
                "flops": 4 * D * c["Hq"] * sum(x * y for x, y in zip(a, b))}
    page = c["page"]
    if c["do"] == "extend":
        pages = sum(-(-(n + o) // page) - -(-o // page) for n, o in zip(a, b))
        # (a new token's old page, where it has one, is read too)
        return {"bytes": 16 * c["S"] + 8 * pages + (8 * sum(a) + 4 * sum(n > 0 and o % page > 0 for n, o in zip(a, b))) * c["slots"], "flops": 0}
    return {"bytes": 9 * c["S"] + 8 * sum(-(-o // page) for o, done in zip(a, b) if done), "flops": 0}


# ---------------------------------------------------------------- inputs


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(n):
    at = [0]
    for x in n:
        at.append(at[-1] + x)
    return at


def prepare(c, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    a, b = _lengths(c)
    return _prepare_cross(c, gen, a, b) if c["do"] == "cross" else _prepare_pages(c, gen, a, b)


def _prepare_cross(c, gen, q, k):
    S, Hq, Hkv = c["S"], c["Hq"], c["Hkv"]

    def normal(*shape, gain=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * gain).to(torch.bfloat16)

    k_start = [i * c["k_hi"] for i in range(S)] if c["layout"] == "padded" else _starts(k)[:-1]
    Tk = max(1, S * c["k_hi"] if c["layout"] == "padded" else sum(k))
    T = sum(q) + c["pad"]
    s = {"c": c, "q": q, "k": k, "T": T, "Tk": Tk, "n": sum(q), "q_start": _ints(_starts(q)), "k_start": _ints(k_start), "k_len": _ints(k),
         "starts": k_start}
    # keys with channels of different strength, as projections give them
    gain = torch.rand((Hkv, D), generator=gen, device="cuda") * 1.2 + 0.3
    if c["layout"] == "fused":
        both = normal(Tk, 2, Hkv, D)
        both[:, 0] *= gain.to(torch.bfloat16)
        s["K"], s["V"] = both[:, 0], both[:, 1]
    else:
        s["K"], s["V"] = normal(Tk, Hkv, D, gain=gain), normal(Tk, Hkv, D)
    s["Q"], s["O"] = normal(T, Hq, D, gain=1.3), normal(T, Hq, D)
    s["lse"] = torch.zeros((T, Hq), device="cuda") if c["lse"] else None
    if own:
        from paper_2605_14513_b200 import heart

        s["config"] = heart.make_cross_config(S, T, Tk, Hq, Hkv, max_q=max(q), kv_strides=(2 * Hkv * D, D) if c["layout"] == "fused" else (0, 0))
        s["workspace"] = heart.new_cross_workspace(s["config"])
    return s


def _prepare_pages(c, gen, a, b):
    S, page, extend = c["S"], c["page"], c["do"] == "extend"
    old = b if extend else a
    held = [-(-n // page) for n in old]
    want = [-(-(n + o) // page) for n, o in zip(a, b)] if extend else held
    n_pages = sum(want) + 5
    # pages in use and free ones as a program that has run for a while has them
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    width = max(1, max(want))
    first = _ints(_starts(held)[:-1]).long()
    column = torch.arange(width, device="cuda")
    table = torch.where(column < _ints(held)[:, None], order[(first[:, None] + column).clamp(max=n_pages - 1)], torch.zeros_like(order[:1]))
    free = n_pages - sum(held)
    free_pages = torch.zeros_like(order)
    free_pages[:free] = order[sum(held):]
    s = {"c": c, "kv_len": _ints(old), "table": table.contiguous(), "free_pages": free_pages, "free_count": _ints([free]),
         "kv_len_out": torch.zeros(S, dtype=torch.int32, device="cuda"), "free_count_out": _ints([0]), "a": a, "b": b}
    if extend:
        T = max(1, sum(a) + c["pad"])
        s.update(T=T, new_len=_ints(a), row_start=torch.zeros(S + 1, dtype=torch.int32, device="cuda"),
                 slots=torch.zeros(T, dtype=torch.int64, device="cuda") if c["slots"] else None)
    else:
        s["done"] = torch.tensor(b, dtype=torch.uint8, device="cuda")
    if own:
        from paper_2605_14513_b200 import heart

        s["config"] = heart.make_cache_config(S, s.get("T", S), 8, 8, page, n_pages, width)
        s["workspace"] = heart.new_cache_workspace(s["config"])
    return s


# ---------------------------------------------------------------- plain forms


def _plain_cross(s):
    """All sequences at once, padded to the longest."""
    c = s["c"]
    S, Hq, Hkv, n, L = c["S"], c["Hq"], c["Hkv"], max(s["q"]), max(1, max(s["k"]))
    lens = s["k_len"][:, None]
    row = torch.arange(n, device="cuda", dtype=torch.int32)
    q = s["Q"][(s["q_start"][:-1, None] + row).clamp(max=s["T"] - 1).long()].float()
    q = q.view(S, n, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, D)
    every = torch.arange(L, device="cuda", dtype=torch.int32)
    held = (s["k_start"][:, None] + every).clamp(max=s["Tk"] - 1).long()
    hidden = every >= lens
    p = (q * D ** -0.5) @ s["K"][held].float().permute(0, 2, 3, 1)
    p.masked_fill_(hidden[:, None, None, :], -math.inf)
    top = p.amax(-1, keepdim=True).clamp(min=-1e30)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ s["V"][held].float().transpose(1, 2)) / torch.where(total > 0, total, torch.ones_like(total))
    rows = torch.arange(s["n"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["q_start"], rows, right=True) - 1
    place = rows - s["q_start"][seq]
    s["O"][:s["n"]] = o.view(S, Hkv, n, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(S, n, Hq, D)[seq, place].to(torch.bfloat16)
    if s["lse"] is not None:
        lse = (top + total.log()).view(S, Hkv, n, Hq // Hkv).permute(0, 2, 1, 3).reshape(S, n, Hq)
        s["lse"][:s["n"]] = lse[seq, place]


def _plain_extend(s):
    page, kv_len, new = s["c"]["page"], s["kv_len"], s["new_len"]
    width = s["table"].shape[1]
    held, after = (kv_len + page - 1) // page, (kv_len + new + page - 1) // page
    need = after - held
    before = need.cumsum(0, dtype=torch.int32) - need
    column = torch.arange(width, device="cuda", dtype=torch.int32)
    # the list is a stack: sequences take from its end, one behind the other
    at = s["free_count"] - 1 - (before[:, None] + column - held[:, None])
    fresh = (column >= held[:, None]) & (column < after[:, None])
    s["table"][:] = torch.where(fresh, s["free_pages"][at.clamp(0, s["free_pages"].numel() - 1).long()], s["table"])
    s["row_start"][0] = 0
    s["row_start"][1:] = new.cumsum(0, dtype=torch.int32)
    torch.add(kv_len, new, out=s["kv_len_out"])
    torch.sub(s["free_count"], need.sum(dtype=torch.int32), out=s["free_count_out"])
    if s["slots"] is not None:
        row = torch.arange(s["T"], device="cuda", dtype=torch.int32)
        seq = (torch.searchsorted(s["row_start"], row, right=True) - 1).clamp(max=new.numel() - 1)
        pos = kv_len[seq] + row - s["row_start"][seq]
        slot = s["table"][seq, (pos // page).clamp(max=width - 1)].long() * page + pos % page
        s["slots"][:] = torch.where(row < s["row_start"][-1], slot, torch.full_like(slot, -1))


def _plain_release(s):
    page, kv_len, done = s["c"]["page"], s["kv_len"], s["done"] != 0
    held = torch.where(done, (kv_len + page - 1) // page, torch.zeros_like(kv_len))
    before = held.cumsum(0, dtype=torch.int32) - held
    column = torch.arange(s["table"].shape[1], device="cuda", dtype=torch.int32)
    back = column < held[:, None]
    s["free_pages"][(s["free_count"] + before[:, None] + column)[back].long()] = s["table"][back]
    s["kv_len_out"][:] = torch.where(done, torch.zeros_like(kv_len), kv_len)
    torch.add(s["free_count"], held.sum(dtype=torch.int32), out=s["free_count_out"])


def _own(s):
    from paper_2605_14513_b200 import heart

    if s["c"]["do"] == "cross":
        heart.heart_cross_attn(s["config"], s["Q"], s["K"], s["V"], s["q_start"], s["k_start"], s["k_len"], s["O"], s["workspace"], lse=s["lse"])
    elif s["c"]["do"] == "extend":
        heart.heart_cache_extend(s["config"], s["new_len"], s["kv_len"], s["free_pages"], s["free_count"], s["table"], s["row_start"], s["workspace"],
                                 slots=s["slots"], kv_len_out=s["kv_len_out"], free_count_out=s["free_count_out"])
    else:
        heart.heart_cache_release(s["config"], s["done"], s["kv_len"], s["free_pages"], s["free_count"], s["table"], s["workspace"],
                                  kv_len_out=s["kv_len_out"], free_count_out=s["free_count_out"])


def run(s):
    do = s["c"]["do"]
    if own:
        _own(s)
    else:
        {"cross": _plain_cross, "extend": _plain_extend, "release": _plain_release}[do](s)
    names = {"cross": ("O", "lse"), "extend": ("table", "row_start", "kv_len_out", "free_count_out", "slots"),
             "release": ("free_pages", "kv_len_out", "free_count_out")}[do]
    return {x: s[x] for x in names if s[x] is not None}


# ---------------------------------------------------------------- the definition in 64 bits


def exact(c, seed):
    s = prepare(c, seed)
    if c["do"] != "cross":
        return _exact_pages(c, s)
    O, G = s["O"].double(), c["Hq"] // c["Hkv"]
    lse = None if s["lse"] is None else s["lse"].double()
    at = 0
    for n, first, L in zip(s["q"], s["starts"], s["k"]):
        here = slice(at, at + n)
        at += n
        for h in range(c["Hkv"] if L else 0):
            k, v = s["K"][first:first + L, h].double(), s["V"][first:first + L, h].double()
            for g in range(h * G, h * G + G):
                logits = s["Q"][here, g].double() @ k.T / math.sqrt(D)
                total = torch.logsumexp(logits, -1, keepdim=True)
                O[here, g] = torch.exp(logits - total) @ v
                if lse is not None:
                    lse[here, g] = total[:, 0]
        if not L:
            O[here] = 0
            if lse is not None:
                lse[here] = -math.inf
    return {"O": O} if lse is None else {"O": O, "lse": lse}


def _exact_pages(c, s):
    """Sequence by sequence, on the host."""
    page, table = c["page"], s["table"].cpu()
    free = s["free_pages"].cpu()
    count = int(s["free_count"])
    if c["do"] == "extend":
        slots = torch.full((s["T"],), -1, dtype=torch.int64)
        at, pages = 0, torch.arange(page)
        for i, (n, o) in enumerate(zip(s["a"], s["b"])):
            for j in range(-(-o // page), -(-(n + o) // page)):
                count -= 1
                table[i, j] = free[count]
            own_slots = (table[i].long()[:, None] * page + pages).flatten()
            slots[at:at + n] = own_slots[o:o + n]
            at += n
        out = {"table": table, "row_start": torch.tensor(_starts(s["a"])), "kv_len_out": torch.tensor([n + o for n, o in zip(s["a"], s["b"])]),
               "free_count_out": torch.tensor([count]), "slots": slots}
        return {x: y.to("cuda", s[x].dtype) for x, y in out.items() if s[x] is not None}
    for i, (o, done) in enumerate(zip(s["a"], s["b"])):
        if done:
            n = -(-o // page)
            free[count:count + n] = table[i, :n]
            count += n
    out = {"free_pages": free, "kv_len_out": torch.tensor([0 if done else o for o, done in zip(s["a"], s["b"])]), "free_count_out": torch.tensor([count])}
    return {x: y.to("cuda", s[x].dtype) for x, y in out.items()}
