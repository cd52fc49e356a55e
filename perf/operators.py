"""The operators around a key / value cache held in 8 bits, as cases that can be timed and compared.

  rope     rotary positions of a step's or a prompt's query and key heads
  append   a step's or a chunk's keys (rotated on the way) and values into pages of e4m3 values, one power-of-two
           scale for each page, head and kind (key / value)
  attend   attention of one or more query tokens per row over such pages, and the attention weight that each
           cached token has received so far
  evict    the cached tokens that received the least weight leave; the others close the gaps

Cache: pool float8_e4m3fn [pages, 2, kv heads, block tokens, dims] (0 keys, 1 values) and exps int8 [pages, 2, kv heads];
a value is pool * 2^exps.  Page 0 belongs to nobody: the rest of a row's table points there.  ``run`` computes the plain
forms in elementary torch operations, or, with ``own``, makes the framework's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
E_MIN, E_MAX, TOP = -32, 31, 448.0


def listed():
    def rope(name, T, heads, dim, rot, dtype, far, interleaved=False, scaling="none", factor=1.0):
        return dict(name=name, op="rope", T=T, heads=heads, dim=dim, rot=rot, dtype=dtype, far=far, interleaved=interleaved,
                    scaling=scaling, factor=factor)

    def append(name, rows, lo, hi, n_lo, n_hi, nq=32, nkv=8, dim=128, block=16, dtype="bf16"):
        return dict(name=name, op="append", rows=rows, lo=lo, hi=hi, n_lo=n_lo, n_hi=n_hi, nq=nq, nkv=nkv, dim=dim, block=block, dtype=dtype)

    def attend(name, rows, lo, hi, n_lo=1, n_hi=1, nq=32, nkv=8, dim=128, block=16, dtype="bf16", window=0, mass=False):
        return dict(name=name, op="attend", rows=rows, lo=lo, hi=hi, n_lo=n_lo, n_hi=n_hi, nq=nq, nkv=nkv, dim=dim, block=block,
                    dtype=dtype, window=window, mass=mass)

    def evict(name, rows, lo, hi, keep, nkv=8, dim=128, block=16):
        return dict(name=name, op="evict", rows=rows, lo=lo, hi=hi, keep=keep, nkv=nkv, dim=dim, block=block)

    return [
        # one request's 32 query and 8 key heads in a decode step
        rope("rope_step_b1", 1, 40, 128, 128, "bf16", 4096),
        # a chunk of a long prompt, frequencies stretched by parts for a context 32 times the trained one
        rope("rope_chunk_4096", 4096, 40, 128, 128, "bf16", 131072, scaling="parts", factor=32.0),
        # an odd chunk of a decoder that rotates neighbouring values of half of each head
        rope("rope_part_fp32_1003", 1003, 16, 128, 64, "fp32", 8192, interleaved=True),
        # the benchmark's step of 64 slots: one token each, mostly into pages that others began
        append("append_step_b64", 64, 16, 1024, 1, 1),
        # pieces of three prompts that share a prefill chunk
        append("append_chunk_3", 3, 300, 6000, 300, 1100),
        # one user at a small decoder with heads of 64
        attend("attend_step_b1", 1, 300, 300, nq=16, nkv=8, dim=64, dtype="fp16"),
        # the benchmark's 64 slots at its context lengths
        attend("attend_step_b64", 64, 512, 4096),
        # two very long contexts, few rows, 8 query heads per key head, pages of 64 tokens
        attend("attend_long_b2", 2, 60000, 100003, nq=32, nkv=4, block=64),
        # a step that also accumulates the weights for eviction
        attend("attend_mass_b32", 32, 1000, 4352, mass=True),
        # the rest of three prompts behind what is already cached, one chunk
        attend("attend_chunk_3", 3, 1500, 8192, n_lo=200, n_hi=700),
        # one request over its budget
        evict("evict_b1", 1, 1003, 1003, 512),
        # sixteen long requests cut to a quarter
        evict("evict_b16", 16, 6000, 8192, 2048),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["rope", "append", "attend", "attend", "evict"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    nkv, dim, block = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128]), rng.choice([16, 16, 32, 64])
    nq = nkv * rng.choice([1, 2, 3, 4, 8])
    if op == "rope":
        dim = rng.choice([64, 96, 128])
        return dict(op=op, T=log_int(1, 4096), heads=rng.randint(1, 40), dim=dim, rot=rng.choice([dim, dim, dim // 2]),
                    dtype=rng.choice(["bf16", "fp16", "fp32"]), far=log_int(64, 1 << 20), interleaved=rng.random() < 0.4,
                    scaling=rng.choice(["none", "linear", "base", "parts", "bands"]), factor=rng.choice([2.0, 8.0, 32.0]))
    rows = log_int(1, 64)
    if op == "append":
        n = 1 if rng.random() < 0.5 else log_int(2, max(2, 3000 // rows))
        lo = log_int(n, 4000)
        return dict(op=op, rows=rows, lo=lo, hi=lo + rng.randint(0, 60000 // rows), n_lo=1 if n == 1 else n // 2, n_hi=n, nq=nq, nkv=nkv,
                    dim=dim, block=block, dtype=dtype)
    if op == "attend":
        if rng.random() < 0.7:
            n, hi = rng.choice([1, 1, 1, 2, 5]), log_int(64, 120000 // rows)
            return dict(op=op, rows=rows, lo=max(n, hi // rng.randint(1, 8)), hi=hi, n_lo=1, n_hi=n, nq=nq, nkv=nkv, dim=dim,
                        block=block, dtype=dtype, window=rng.choice([0, 0, 0, 700]), mass=n == 1 and rng.random() < 0.4)
        rows, nkv = rng.randint(1, 4), rng.choice([2, 4])
        n = log_int(16, 800 // rows)
        hi = n + log_int(1, 4000 // rows)
        return dict(op=op, rows=rows, lo=n, hi=hi, n_lo=n // 2, n_hi=n, nq=nkv * rng.choice([2, 4, 8]), nkv=nkv, dim=dim, block=block,
                    dtype=dtype, window=rng.choice([0, 0, 500]), mass=False)
    hi = log_int(200, 100000 // rows)
    return dict(op=op, rows=rows, lo=max(8, hi // 2), hi=hi, keep=max(64, hi // rng.randint(2, 6)), nkv=nkv, dim=dim, block=block)


# ---- what a program has in hand before the call ----

def _ragged(case):
    """Cached tokens of every row (its new ones among them) and its new tokens: host lists, the case's own."""
    g = torch.Generator().manual_seed(case["rows"] + 7 * case["lo"])
    ints = lambda lo, hi: torch.randint(lo, hi + 1, (case["rows"],), generator=g).tolist()
    n = ints(case.get("n_lo", 1), case.get("n_hi", 1))
    return [max(a, b) for a, b in zip(ints(case["lo"], case["hi"]), n)], n


def _frequencies(rot, theta, scaling, factor, original, low, high):
    """Angle per position of every pair, 64 bits, and what the rotated values are multiplied by."""
    i = torch.arange(rot // 2, dtype=torch.float64)
    base, m = theta, 1.0
    if scaling == "base":
        base = theta * factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":      # pairs that turn fewer than `low` times in the trained context are stretched, above `high` times not
        where = lambda turns: rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(theta))
        first, last = max(math.floor(where(high)), 0), min(math.ceil(where(low)), rot - 1)
        ramp = ((i - first) / max(last - first, 1e-3)).clamp(0, 1)
        f, m = f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1.0
    elif scaling == "bands":      # the same by wavelength, without a change of magnitude
        s = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f / factor * (1 - s) + f * s
    return f, m


def _rope_options(case):
    original = 4096
    high = {"parts": 32.0, "bands": 4.0}.get(case.get("scaling"), 1.0)
    return dict(rot_dim=case.get("rot", case["dim"]), theta=1000000.0, interleaved=case.get("interleaved", False),
                scaling=case.get("scaling", "none"), factor=case.get("factor", 1.0), original_context=original, low=1.0, high=high)


def _e_of(amax):
    """Smallest e with amax <= 448 * 2^e = 0.875 * 2^(9 + e), within its range."""
    m, x = torch.frexp(amax)
    return (x - 9 + (m > 0.875).to(x.dtype)).clamp(E_MIN, E_MAX).where(amax > 0, torch.full_like(x, E_MIN))


def _to8(x, e):
    return torch.ldexp(x, -e).clamp(-TOP, TOP).to(torch.float8_e4m3fn)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    s = dict(case=case)
    opt = _rope_options(case)
    if case["op"] in ("rope", "append"):
        f, s["magnitude"] = _frequencies(opt["rot_dim"], opt["theta"], opt["scaling"], opt["factor"], opt["original_context"],
                                         opt["low"], opt["high"])
        s["freq"] = f.cuda()
    if case["op"] == "rope":
        dt = DTYPES[case["dtype"]]
        # the heads are the front part of a wider projection
        s["x"] = (normal(case["T"], case["heads"] + 2, case["dim"]) * 1.28).to(dt)[:, :case["heads"]]
        first = torch.randint(0, max(1, case["far"] - case["T"]), (1,), generator=g, device="cuda", dtype=torch.int32)
        s["pos"] = first + torch.arange(case["T"], device="cuda", dtype=torch.int32)
        if own:
            from paper_2608_14376_b200 import corun
            s["rope"], s["y"] = corun.Rope(**opt), torch.empty(s["x"].shape, dtype=dt, device="cuda")
        return s
    B, nkv, dim, block = case["rows"], case["nkv"], case["dim"], case["block"]
    ctx, n = _ragged(case)
    per_row = -(-max(ctx) // block)
    pages = sum(-(-c // block) for c in ctx) + 1
    order = torch.randperm(pages - 1, generator=g, device="cuda").to(torch.int32) + 1
    table = torch.zeros(B, per_row, dtype=torch.int32, device="cuda")
    at = 0
    for b, c in enumerate(ctx):
        k = -(-c // block)
        table[b, :k] = order[at:at + k]
        at += k
    x = normal(pages, 2, nkv, block, dim) * 1.28 * torch.exp(0.3 * normal(pages, 2, nkv, 1, 1))
    x[:, 0] *= 0.5 + 1.5 * torch.rand(nkv, 1, dim, generator=g, device="cuda")       # some key channels are larger than others
    e = _e_of(x.abs().amax((-1, -2)))
    s["pool"], s["exps"] = _to8(x, e[..., None, None]), e.to(torch.int8)
    del x
    s["table"], s["ctx"] = table, torch.tensor(ctx, dtype=torch.int32, device="cuda")
    T = sum(n)
    s["T"], s["max_new"] = T, max(n)
    s["cu"] = torch.tensor([0] + n, device="cuda").cumsum(0).to(torch.int32) if case.get("n_hi", 1) > 1 else None
    if case["op"] == "append":
        dt = DTYPES[case["dtype"]]
        qkv = (normal(T, case["nq"] + 2 * nkv, dim) * 1.28).to(dt)                    # the fused projection
        s["q"], s["k"], s["v"] = qkv.split([case["nq"], nkv, nkv], 1)
        row = torch.repeat_interleave(torch.arange(B), torch.tensor(n))
        s["pos"] = torch.tensor([c - m + i for c, m in zip(ctx, n) for i in range(m)], dtype=torch.int32, device="cuda")
        s["row"] = row.cuda()
    elif case["op"] == "attend":
        dt = DTYPES[case["dtype"]]
        s["q"] = (normal(T, case["nq"], dim) * 1.5).to(dt)
        s["scale"] = dim ** -0.5
        s["row"] = torch.repeat_interleave(torch.arange(B), torch.tensor(n)).cuda()
        last = s["table"].gather(1, ((s["ctx"].long() - 1) // block)[:, None])[:, 0].long()
        off = torch.arange(block, device="cuda")
        # what lies behind a row's last token in its last page is whatever the page held before: not numbers
        behind = (off[None] > ((s["ctx"] - 1) % block)[:, None])[:, None, None, :, None]
        bits = s["pool"].view(torch.uint8)
        bits[last] = torch.where(behind, torch.full_like(bits[last], 0x7F), bits[last])
        s["out"] = torch.zeros(T, case["nq"], dim, dtype=dt, device="cuda")
    if case["op"] == "evict" or case.get("mass"):
        s["mass"] = torch.rand(B, nkv, per_row * block, generator=g, device="cuda") ** 6 * 5.0     # few tokens hold most of it
        s["mass"][..., ::7] = s["mass"][..., :1]                                                    # ties
    if case["op"] == "evict":
        s["keep"] = torch.full((B,), case["keep"], dtype=torch.int32, device="cuda")
        s["sinks"], s["recent"] = 4, case["keep"] // 4
    if own:
        from paper_2608_14376_b200 import corun
        s["cache"] = corun.Kv8Cache(pages, nkv, dim, block, pool=s["pool"], exps=s["exps"])
        if case["op"] == "append":
            s["rope"] = corun.Rope(**opt)
            s["q_out"] = torch.empty(T, case["nq"], dim, dtype=dt, device="cuda")
        if case["op"] == "attend":
            s["attention"] = corun.Kv8Attention(B, case["nq"], nkv, dim, per_row, block, tokens=T, max_new=s["max_new"])
    return s


# ---- plain forms ----

def _rotate(x, pos, freq, magnitude, interleaved):
    """x [T, heads, dim]: its first 2 * len(freq) dims rotated, 32 bits; angles in 64 bits (positions reach a million)."""
    rot = 2 * freq.numel()
    a = pos.double()[:, None] * freq
    c, s = (a.cos() * magnitude).float()[:, None], (a.sin() * magnitude).float()[:, None]
    x = x.float()
    h, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        x1, x2 = h[..., 0::2], h[..., 1::2]
        y = torch.stack((x1 * c - x2 * s, x2 * c + x1 * s), -1).flatten(-2)
    else:
        x1, x2 = h[..., :rot // 2], h[..., rot // 2:]
        y = torch.cat((x1 * c - x2 * s, x2 * c + x1 * s), -1)
    return torch.cat((y, rest), -1)


def _append(s):
    block, pool, exps, table, ctx = s["case"]["block"], s["pool"], s["exps"], s["table"], s["ctx"].long()
    k = _rotate(s["k"], s["pos"], s["freq"], s["magnitude"], False)
    q = _rotate(s["q"], s["pos"], s["freq"], s["magnitude"], False).to(s["q"].dtype)
    kv = torch.stack((k, s["v"].float()), 1)                                   # [T, 2, kv heads, dim]
    T, row = s["T"], s["row"]
    cu = s["cu"].long() if s["cu"] is not None else torch.arange(len(ctx) + 1, device=ctx.device)
    start = ctx - (cu[1:] - cu[:-1])                                           # first new index of every row
    index = start[row] + torch.arange(T, device=ctx.device) - cu[row]
    page, off = table[row, index // block].long(), index % block
    # the largest magnitude that arrives in every page, and the page's old scale where it was begun before
    amax = torch.zeros(exps.shape, device=ctx.device).index_reduce_(0, page, kv.abs().amax(-1), "amax")
    begun = start % block                                                      # old tokens in the first page of every row
    first = table.gather(1, (start // block).clamp(max=table.shape[1] - 1)[:, None])[:, 0].long()
    begun_page = torch.zeros(len(exps), dtype=torch.bool, device=ctx.device).index_fill_(0, first, True)
    begun_page &= torch.zeros(len(exps), dtype=torch.long, device=ctx.device).index_put_((first,), begun) > 0
    e = _e_of(amax)
    e = torch.where(begun_page[:, None, None], torch.maximum(e, exps.int()), e)
    # old tokens of begun pages move to the new scale
    old = pool[first]
    moved = _to8(old.float(), (e[first] - exps[first].int())[..., None, None])
    is_old = (torch.arange(block, device=ctx.device)[None] < begun[:, None])[:, None, None, :, None]
    bits = pool.view(torch.uint8)
    bits[first] = torch.where(is_old, moved.view(torch.uint8), old.view(torch.uint8))
    bits[page, :, :, off] = _to8(kv, e[page][..., None]).view(torch.uint8)
    exps[page] = e[page].to(torch.int8)
    return {"q": q, "pool": pool, "exps": exps}


def _padded(s):
    """Ragged query tokens as [rows, most]: their places in q, and where there is one."""
    B, most = s["case"]["rows"], s["max_new"]
    cu = s["cu"].long() if s["cu"] is not None else torch.arange(B + 1, device="cuda")
    i = torch.arange(most, device="cuda")
    n = cu[1:] - cu[:-1]
    return (cu[:-1, None] + i).clamp(max=s["T"] - 1), n, i, cu


def _attend(s):
    case = s["case"]
    B, nkv, G, dim, block = case["rows"], case["nkv"], case["nq"] // case["nkv"], case["dim"], case["block"]
    at, n, i, cu = _padded(s)
    S = s["table"].shape[1] * block
    t = torch.arange(S, device="cuda")
    lim = s["ctx"].long()[:, None] - n[:, None] + i                            # last visible index of every query
    see = (t <= lim[..., None]) & (i < n[:, None])[..., None]                  # [B, most, S]
    if case["window"]:
        see &= t > lim[..., None] - case["window"]
    live = (t < s["ctx"][:, None])[:, None, :, None]
    page = s["table"].long()
    kv = torch.ldexp(s["pool"][page].float(), s["exps"][page].int()[..., None, None])   # [B, pages, 2, kv heads, block, dim]
    k, v = (kv[:, :, j].permute(0, 2, 1, 3, 4).reshape(B, nkv, S, dim) for j in (0, 1))
    q = s["q"].float()[at].reshape(B, len(i), nkv, G, dim).permute(0, 2, 1, 3, 4).reshape(B, nkv, -1, dim)
    x = (q @ k.transpose(-1, -2)).view(B, nkv, len(i), G, S) * s["scale"]
    see = see[:, None, :, None]
    x = torch.where(see, x, torch.full_like(x, -math.inf))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top.isfinite(), top, torch.zeros_like(top)))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = p.reshape(B, nkv, -1, S) @ torch.where(live, v, torch.zeros_like(v))
    o = o.view(B, nkv, len(i), G, dim).permute(0, 2, 1, 3, 4).reshape(B, len(i), nkv * G, dim)
    s["out"].copy_(o[s["row"], torch.arange(s["T"], device="cuda") - cu[s["row"]]])
    if not case["mass"]:
        return {"out": s["out"]}
    s["mass"] += p.sum((2, 3))
    return {"out": s["out"], "mass": s["mass"]}


def _evict(s):
    case, mass, ctx = s["case"], s["mass"], s["ctx"].long()
    B, nkv, block, most = case["rows"], case["nkv"], case["block"], case["keep"]
    S = mass.shape[-1]
    t = torch.arange(S, device="cuda")
    cut = (s["keep"] > 0) & (s["keep"] < s["ctx"])
    valid = t < ctx[:, None]
    safe = valid & ((t < s["sinks"]) | (t >= ctx[:, None] - s["recent"]))
    score = torch.where(valid[:, None], mass, torch.full_like(mass, -math.inf))
    score = torch.where(safe[:, None], torch.full_like(mass, math.inf), score)
    rank = torch.argsort(score, dim=-1, descending=True, stable=True)                     # the lowest index first among equals
    place = torch.empty_like(rank).scatter_(-1, rank, t.expand_as(rank))
    stays = place < s["keep"][:, None, None]
    src = torch.where(stays, t, S).sort(-1).values[..., :most]                 # [B, kv heads, keep] in order
    live = (src < S) & cut[:, None, None]
    src = torch.where(live, src, 0)
    page = s["table"].long()
    b, h = torch.arange(B, device="cuda")[:, None, None], torch.arange(nkv, device="cuda")[:, None]
    from_page, from_off = page[b, src // block], src % block
    e_src = s["exps"][from_page, :, h].int()                                   # [B, kv heads, keep, 2]
    data = s["pool"].view(torch.uint8)[from_page, :, h, from_off].view(torch.float8_e4m3fn)     # [B, kv heads, keep, 2, dim]
    blocks = -(-most // block)
    pad = torch.nn.functional.pad(torch.where(live[..., None], e_src, E_MIN), (0, 0, 0, blocks * block - most), value=E_MIN)
    e_new = pad.view(B, nkv, blocks, block, 2).amax(3)                          # [B, kv heads, blocks, 2]
    e_tok = e_new.repeat_interleave(block, 2, output_size=blocks * block)[:, :, :most]
    data = _to8(data.float(), (e_tok - e_src)[..., None]).view(torch.uint8)
    # rows that stay as they are write what page 0 holds to page 0
    dst = torch.arange(most, device="cuda")
    to_page = torch.where(live, page[b, dst // block], 0)
    bits = s["pool"].view(torch.uint8)
    data = torch.where(live[..., None, None], data, bits[0, :, :, 0].transpose(0, 1)[None, :, None])
    bits[to_page, :, h, torch.where(live, dst % block, 0)] = data
    begun = torch.where(live.any(-1)[..., None], page[b, torch.arange(blocks, device="cuda")], 0)
    s["exps"][begun, :, h] = torch.where(live.any(-1)[..., None, None], e_new, s["exps"][0].T[None, :, None].int()).to(torch.int8)
    moved = mass.gather(-1, src)
    mass[..., :most] = torch.where(live, moved, mass[..., :most])
    return {"kept": torch.where(live, src, -1).int(), "ctx": torch.where(cut, s["keep"], s["ctx"]), "pool": s["pool"],
            "exps": s["exps"], "mass": mass}


def run(state):
    s, case = state, state["case"]
    if own:
        if case["op"] == "rope":
            return s["rope"].apply(s["x"], s["pos"], out=s["y"])
        if case["op"] == "append":
            q = s["cache"].append(s["k"], s["v"], s["ctx"], s["table"], cu=s["cu"], positions=s["pos"], rope=s["rope"], q=s["q"],
                                  q_out=s["q_out"])
            return {"q": q, "pool": s["pool"], "exps": s["exps"]}
        if case["op"] == "attend":
            out = s["attention"].run(s["q"], s["cache"], s["ctx"], s["table"], s["scale"], cu=s["cu"], window=case["window"],
                                     mass=s.get("mass"), out=s["out"])
            return {"out": out, "mass": s["mass"]} if case["mass"] else {"out": out}
        kept, ctx = s["cache"].evict(s["ctx"], s["table"], s["mass"], s["keep"], case["keep"], sinks=s["sinks"], recent=s["recent"])
        return {"kept": kept, "ctx": ctx, "pool": s["pool"], "exps": s["exps"], "mass": s["mass"]}
    if case["op"] == "rope":
        return _rotate(s["x"], s["pos"], s["freq"], s["magnitude"], case["interleaved"]).to(s["x"].dtype)
    return {"append": _append, "attend": _attend, "evict": _evict}[case["op"]](s)


def work(case):
    size = 4 if case.get("dtype") == "fp32" else 2
    if case["op"] == "rope":
        n = case["T"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * size + 4 * case["T"], "flops": 3 * case["T"] * case["heads"] * case["rot"]}
    ctx, n = _ragged(case)
    nkv, dim, block = case["nkv"], case["dim"], case["block"]
    if case["op"] == "append":
        T = sum(n)
        begun = sum((c - m) % block for c, m in zip(ctx, n))                   # old tokens, read and written where a scale grows
        return {"bytes": T * (2 * case["nq"] + 2 * nkv) * dim * size + 2 * T * nkv * dim + 2 * begun * nkv * dim,
                "flops": 3 * T * (case["nq"] + nkv) * dim + 2 * T * nkv * dim}
    if case["op"] == "attend":
        read = sum(min(c, case["window"] + m - 1) if case["window"] else c for c, m in zip(ctx, n))
        pairs = sum(min(c - m + i + 1, case["window"] or c) for c, m in zip(ctx, n) for i in range(m))
        return {"bytes": read * nkv * 2 * dim + 2 * sum(n) * case["nq"] * dim * size + (8 * sum(ctx) * nkv if case["mass"] else 0),
                "flops": 4 * pairs * case["nq"] * dim}
    kept = sum(min(c, case["keep"]) for c in ctx if c > case["keep"])
    return {"bytes": nkv * (4 * sum(ctx) + kept * (4 * dim + 4 + 4 + 4)), "flops": nkv * sum(ctx)}


# ---- the operators' definition in 64 bits ----

def _turned(x, pos, freq, magnitude, interleaved):
    """The pairs as complex numbers, multiplied by magnitude * exp(i pos freq)."""
    rot = 2 * freq.numel()
    x = x.double()
    h = x[..., :rot]
    z = torch.view_as_complex(h.unflatten(-1, (-1, 2)).contiguous() if interleaved else h.unflatten(-1, (2, -1)).transpose(-1, -2).contiguous())
    a = (pos.double()[:, None] * freq)[:, None]
    z = torch.view_as_real(z * torch.polar(torch.full_like(a, magnitude), a))
    return torch.cat((z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2), x[..., rot:]), -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _turned(s["x"], s["pos"], s["freq"], s["magnitude"], case["interleaved"])
    if case["op"] == "append":
        # which of two neighbouring 8-bit values a key becomes hangs on its last bit where it lies between them: no value for the pool
        return {"q": _turned(s["q"], s["pos"], s["freq"], s["magnitude"], False), "pool": None, "exps": None}
    if case["op"] == "evict":
        return None
    block, nkv, G = case["block"], case["nkv"], case["nq"] // case["nkv"]
    ctx, n = _ragged(case)
    out, first = [], 0
    mass = s["mass"].double() if case["mass"] else None
    for b, (c, m) in enumerate(zip(ctx, n)):
        page = s["table"][b, :-(-c // block)].long()
        kv = s["pool"][page].double() * 2.0 ** s["exps"][page].double()[..., None, None]
        k, v = kv.transpose(1, 3).flatten(0, 1)[:c].permute(2, 1, 0, 3)        # 2 x [kv heads, c, dim]
        q = s["q"][first:first + m].double().unflatten(1, (nkv, G)) * s["scale"]
        x = torch.einsum("mhgd,htd->hgmt", q, k)
        d = torch.arange(c - m, c, device="cuda")[:, None] - torch.arange(c, device="cuda")
        hidden = (d < 0) | (d >= case["window"]) if case["window"] else d < 0
        p = x.masked_fill(hidden, -math.inf).softmax(-1)
        out.append(torch.einsum("hgmt,htd->mhgd", p, v).flatten(1, 2))
        if mass is not None:
            mass[b, :, :c] += p.sum((1, 2))
        first += m
    return {"out": torch.cat(out), **({"mass": mass} if mass is not None else {})}
