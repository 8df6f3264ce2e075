"""What stands before and behind the pre-filling of a prompt, as timing cases: rotary positions of its queries and
keys, the page bookkeeping of the requests that go on from it, their new keys and values written into the pages, and the
attention of all these requests to the prompt that they share and to what each has of its own.

A case's "op" names the operator:
  rotary  queries and keys rotated by their positions, or the gradients rotated back
  table   block tables, slot maps and positions of one step, from the requests' lengths
  append  a step's queries and keys rotated, keys and values written into their pages
  prefix  attention to a shared contiguous prefix and to paged suffixes
Lengths of requests follow from the case alone ("lens_seed"), everything else from the seed.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


# --- cases ----------------------------------------------------------------------------------------------

def _rotary(name, tokens, *, hq=32, hkv=8, d=128, rot=128, layout="half", scaling="bands", theta=500000.0, start=0,
            seqs=1, dtype="bf16", backward=False):
    return _named(name, {"op": "rotary", "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "rot": rot, "layout": layout,
                         "scaling": scaling, "theta": theta, "start": start, "seqs": seqs, "dtype": dtype,
                         "backward": backward})


def _table(name, requests, *, page=64, most_past=4096, most_new=1, finished=0.0, offset=0, lens_seed=1):
    return _named(name, {"op": "table", "requests": requests, "page": page, "most_past": most_past,
                         "most_new": most_new, "finished": finished, "offset": offset, "lens_seed": lens_seed})


def _append(name, requests, *, hq=32, hkv=8, d=128, rot=128, layout="half", page=64, most_past=1024, most_new=1,
            padding=0, offset=131072, dtype="bf16", lens_seed=1):
    return _named(name, {"op": "append", "requests": requests, "hq": hq, "hkv": hkv, "d": d, "rot": rot,
                         "layout": layout, "page": page, "most_past": most_past, "most_new": most_new,
                         "padding": padding, "offset": offset, "dtype": dtype, "scaling": "bands", "theta": 500000.0,
                         "lens_seed": lens_seed})


def _prefix(name, requests, prefix, *, hq=32, hkv=8, d=128, page=64, most_past=1024, most_new=1, padding=0, lse=False,
            dtype="bf16", lens_seed=1):
    return _named(name, {"op": "prefix", "requests": requests, "prefix": prefix, "hq": hq, "hkv": hkv, "d": d,
                         "page": page, "most_past": most_past, "most_new": most_new, "padding": padding, "lse": lse,
                         "dtype": dtype, "lens_seed": lens_seed})


def _named(name, case):
    return {"name": name, **case} if name else case


def listed():
    return [
        # One new token far into a long context: a single user's decoding step, nothing but latency.
        _rotary("rotary_1_token", 1, start=131072),
        # The headline layer's whole prompt before it is pre-filled.
        _rotary("rotary_128k", 131072),
        # Packed prompts of an odd total, half of each head rotated in neighbouring pairs, in fp16.
        _rotary("rotary_packed_part", 40961, hq=28, hkv=4, rot=64, layout="interleaved", scaling="none",
                theta=10000.0, seqs=7, dtype="fp16"),
        # The gradients of a long training sequence, in fp32, positions stretched beyond the trained length.
        _rotary("rotary_backward_32k", 32768, scaling="yarn", theta=1000000.0, dtype="fp32", backward=True),
        # The page bookkeeping of a decoding step: every request has one new token, few need a new page.
        _table("table_decode", 64, offset=131072),
        # A step of a busy server: new prompts beside decoding requests, finished ones give their pages back.
        _table("table_mixed", 1000, page=16, most_past=3000, most_new=700, finished=0.1),
        # New keys and values of a decoding step go to their pages.
        _append("append_decode", 64),
        # Follow-up prompts of different lengths behind a shared prefix, the batch padded to a round size.
        _append("append_prompts", 48, hq=28, hkv=4, most_new=1500, padding=123, page=16),
        # A short system prompt and a handful of requests on a small model: launches and latency.
        _prefix("prefix_small", 4, 1000, hq=8, hkv=2, d=64, page=16, most_past=64),
        # Questions on one document: ordinary serving, bound by reading the document's keys and values once.
        _prefix("prefix_decode_32k", 16, 32768, most_past=2000, lse=True),
        # Many samples from the headline prompt: as much arithmetic as memory traffic.
        _prefix("prefix_decode_128k", 64, 131072, most_past=700),
        # Drafted tokens checked by a model of seven query heads per KV head: several tokens per request, causal among
        # themselves, a padded batch, an odd prefix, fp16.
        _prefix("prefix_drafts_64k", 24, 65535, hq=28, hkv=4, page=16, most_past=1200, most_new=8, padding=5,
                dtype="fp16", lse=True),
    ]


HEADS = [(32, 8), (28, 4), (32, 8), (28, 4), (16, 8), (8, 1), (4, 4), (1, 1)]


def _between(rng, lo, hi):
    """A whole number, spread over the logarithm of the range."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most[c["op"]] = max(most.get(c["op"], 0.0), w["bytes"], w["flops"] / 50)
    while True:
        op = rng.choice(["rotary", "rotary", "table", "append", "prefix", "prefix", "prefix"])
        hq, hkv = rng.choice(HEADS)
        d = rng.choice([128, 128, 64, 256])
        seed = rng.randrange(1 << 20)
        page = rng.choice([16, 32, 64, 128])
        if op == "rotary":
            rot = rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)])
            case = _rotary("", _between(rng, 1, 131072), hq=hq, hkv=hkv, d=d, rot=rot,
                           layout=rng.choice(["half", "interleaved"]),
                           scaling=rng.choice(["none", "linear", "ntk", "yarn", "bands"]) if rot > 2 else "none",
                           theta=rng.choice([10000.0, 500000.0, 1000000.0]), start=rng.choice([0, rng.randrange(1 << 20)]),
                           seqs=rng.choice([1, 1, rng.randint(1, 9)]), dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                           backward=rng.random() < 0.3)
        elif op == "table":
            case = _table("", _between(rng, 1, 1000), page=page, most_past=_between(rng, 1, 8000),
                          most_new=rng.choice([1, _between(rng, 1, 700)]), finished=rng.choice([0.0, 0.1, 0.5]),
                          offset=rng.choice([0, rng.randrange(1 << 17)]), lens_seed=seed)
        elif op == "append":
            case = _append("", _between(rng, 1, 200), hq=hq, hkv=hkv, d=d, rot=rng.choice([d, d // 2]),
                           layout=rng.choice(["half", "interleaved"]), page=page, most_past=_between(rng, 1, 2000),
                           most_new=rng.choice([1, _between(rng, 1, 1500)]), padding=rng.choice([0, rng.randint(1, 99)]),
                           dtype=rng.choice(["bf16", "bf16", "fp16"]), lens_seed=seed)
        else:
            case = _prefix("", _between(rng, 1, 64), _between(rng, 1, 131072), hq=hq, hkv=hkv, d=d, page=page,
                           most_past=_between(rng, 1, 3000), most_new=rng.choice([1, 1, rng.randint(1, 16)]),
                           padding=rng.choice([0, 0, rng.randint(1, 9)]), lse=rng.random() < 0.5,
                           dtype=rng.choice(["bf16", "bf16", "fp16"]), lens_seed=seed)
            if _tokens(case) * hq * case["prefix"] > 1 << 28:   # the plain form's scores: 1 GiB
                continue
        w = work(case)
        if max(w["bytes"], w["flops"] / 50) <= most[op]:
            return case


def _lens(case):
    """Tokens that each request has in its pages, and new ones of this step (-1: it has finished)."""
    r = random.Random(case["lens_seed"])
    past = [r.randint(0, case["most_past"]) for _ in range(case["requests"])]
    new = [r.randint(1, case["most_new"]) if case["most_new"] > 1 else 1 for _ in range(case["requests"])]
    if case["most_new"] > 1 and case["requests"] > 2:
        new[r.randrange(case["requests"])] = 0                  # a request that waits this step
    if case["op"] == "table":
        new = [-1 if r.random() < case["finished"] else n for n in new]
    return past, new


def _tokens(case):
    """Rows of the step's tensors: the new tokens, and what the batch is padded with."""
    return sum(max(n, 0) for n in _lens(case)[1]) + case.get("padding", 0)


def _pages(n, page):
    return -(-n // page)


def work(case):
    size = BYTES[case["dtype"]] if "dtype" in case else 4
    if case["op"] == "rotary":
        values = case["tokens"] * (case["hq"] + case["hkv"])
        return {"bytes": 2 * size * values * case["d"] + 4 * case["tokens"] + 4 * case["rot"],
                "flops": 3 * values * case["rot"]}
    past, new = _lens(case)
    tokens, page = sum(max(n, 0) for n in new), case["page"]
    if case["op"] == "table":
        moved = sum(_pages(p + n, page) - _pages(p, page) if n >= 0 else _pages(p, page) for p, n in zip(past, new))
        return {"bytes": 4 * (4 * case["requests"] + 2 * moved + 2 * tokens), "flops": 4 * case["requests"] + 4 * tokens}
    if case["op"] == "append":
        return {"bytes": 2 * size * tokens * (case["hq"] + 2 * case["hkv"]) * case["d"] + 8 * tokens,
                "flops": 3 * tokens * (case["hq"] + case["hkv"]) * case["rot"]}
    keys = case["prefix"] + sum(p + n for p, n in zip(past, new))
    pairs = tokens * case["prefix"] + sum(n * p + n * (n + 1) // 2 for p, n in zip(past, new))
    return {"bytes": size * case["d"] * (2 * keys * case["hkv"] + 2 * tokens * case["hq"]),
            "flops": 4 * case["d"] * case["hq"] * pairs}


# --- inputs ---------------------------------------------------------------------------------------------

def _turns(case):
    """Turns per position of each pair of rotary dimensions, and the factor on the rotated values."""
    r, theta, kind = case["rot"], case["theta"], case["scaling"]
    factor, trained = 8.0, 8192.0
    if kind == "ntk":
        theta *= factor ** (r / (r - 2))
    freq = [theta ** (-2.0 * i / r) for i in range(r // 2)]
    if kind == "linear":
        freq = [f / factor for f in freq]
    elif kind == "yarn":
        def dim(rotations):
            return r * math.log(trained / (rotations * 2 * math.pi)) / (2 * math.log(theta))
        lo, hi = max(math.floor(dim(32.0)), 0), min(math.ceil(dim(1.0)), r - 1)
        ramp = [min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(r // 2)]
        freq = [f * (1 - x) + f / factor * x for f, x in zip(freq, ramp)]
    elif kind == "bands":
        low, high = 1.0, 4.0
        keep = [min(max((trained * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for f in freq]
        freq = [f / factor * (1 - x) + f * x for f, x in zip(freq, keep)]
    return [f / (2 * math.pi) for f in freq], (0.1 * math.log(factor) + 1.0 if kind == "yarn" else 1.0)


def _whole(values, dev):
    return torch.tensor(values, dtype=torch.int32, device=dev)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    s = {"op": case["op"], "case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32).to(TYPES[case["dtype"]])

    if case["op"] in ("rotary", "append"):
        turns, s["factor"] = _turns(case)
        s["turns"] = torch.tensor(turns, dtype=torch.float64, device=dev)
    if case["op"] == "rotary":
        T, n = case["tokens"], _pages(case["tokens"], case["seqs"])
        s["positions"] = (torch.arange(T, device=dev) % n + case["start"]).to(torch.int32)
        s["q"], s["k"] = normal(T, case["hq"], case["d"]), normal(T, case["hkv"], case["d"])
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        return s

    past, new = _lens(case)
    R, P = case["requests"], case["page"]
    held = [_pages(p, P) for p in past]
    most = max(_pages(p + max(n, 0), P) for p, n in zip(past, new)) + 3     # entries of a table row
    T = _tokens(case)
    if case["op"] == "table":
        # half as many free pages again as the step needs, somewhere in the ring
        free = sum(_pages(p + max(n, 0), P) - h for p, n, h in zip(past, new, held)) * 3 // 2 + 8
        pages = sum(held) + free
        order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
        first = torch.tensor(held, device=dev).cumsum(0) - torch.tensor(held, device=dev)
        at = torch.arange(most, device=dev)
        own_page = at[None, :] < torch.tensor(held, device=dev)[:, None]
        s["table"] = torch.where(own_page, order[(first[:, None] + at[None, :]).clamp(max=pages - 1)], -1).contiguous()
        head = int(torch.randint(pages, (1,), generator=g, device=dev))
        s["ring"] = torch.full((pages,), -1, dtype=torch.int32, device=dev)
        s["ring"][(torch.arange(free, device=dev) + head) % pages] = order[sum(held):]
        s["ring_state"] = _whole([head, free], dev)
        s["past"], s["new"] = _whole(past, dev), _whole(new, dev)
        s["capacity"] = T + 17                                              # a padded batch
        s["lens"], s["ring_state_out"], s["cu"] = (torch.empty(n, dtype=torch.int32, device=dev) for n in (R, 2, R + 1))
        s["positions"], s["slots"] = (torch.empty(s["capacity"], dtype=torch.int32, device=dev) for _ in range(2))
        s["status"] = torch.empty(4, dtype=torch.int32, device=dev)
        return s

    total = [p + n for p, n in zip(past, new)]
    need = [_pages(n, P) for n in total]
    pages = sum(need) + 5
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    first = torch.tensor(need, device=dev).cumsum(0) - torch.tensor(need, device=dev)
    at = torch.arange(most, device=dev)
    own_page = at[None, :] < torch.tensor(need, device=dev)[:, None]
    s["table"] = torch.where(own_page, order[(first[:, None] + at[None, :]).clamp(max=pages - 1)], -1).contiguous()
    s["lens"] = _whole(total, dev)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    s["cu"] = _whole(cu, dev)
    s["k_pages"], s["v_pages"] = (normal(pages, P, case["hkv"], case["d"]) for _ in range(2))
    s["q"] = normal(T, case["hq"], case["d"])
    if case["op"] == "append":
        s["k"], s["v"] = normal(T, case["hkv"], case["d"]), normal(T, case["hkv"], case["d"])
        owner = torch.repeat_interleave(torch.arange(R, device=dev), torch.tensor(new, device=dev))
        place = torch.arange(cu[-1], device=dev) - s["cu"].long()[owner] + torch.tensor(past, device=dev)[owner]
        s["slots"] = torch.full((T,), -1, dtype=torch.int32, device=dev)
        s["slots"][:cu[-1]] = (s["table"].long()[owner, place // P] * P + place % P).to(torch.int32)
        s["positions"] = torch.zeros(T, dtype=torch.int32, device=dev)
        s["positions"][:cu[-1]] = (place + case["offset"]).to(torch.int32)
        s["q_out"] = normal(T, case["hq"], case["d"])                       # what padding rows keep
        return s

    # keys and queries with a common part, and a first key that every query looks at
    L, G = case["prefix"], case["hq"] // case["hkv"]
    s["prefix_k"], s["prefix_v"] = normal(L, case["hkv"], case["d"]), normal(L, case["hkv"], case["d"])
    common = normal(case["hkv"], case["d"])
    s["q"] = (s["q"].view(T, case["hkv"], G, case["d"]) + 0.5 * common[:, None, :]).view(T, case["hq"], case["d"])
    s["prefix_k"][0] = 2.0 * common
    s["scale"] = case["d"] ** -0.5
    s["out"] = normal(T, case["hq"], case["d"])                             # what padding rows keep
    s["lse"] = torch.zeros(case["hq"], T, dtype=torch.float32, device=dev) if case["lse"] else None
    s["max_new"] = max(max(new), 1)
    s["max_suffix"] = most * P
    if case["most_new"] == 1 and not case["padding"]:
        s["cu"] = None                                                      # one token per request
    return s


# --- one pass -------------------------------------------------------------------------------------------

def run(state):
    return (OWN if own else PLAIN)[state["op"]](state)


def _turned(x, cos, sin, rot, layout):
    """x [T, H, d] in fp32, cos and sin [T, rot / 2]."""
    c, n = cos[:, None, :], sin[:, None, :]
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * c - b * n, b * c + a * n, x[..., rot:]], dim=-1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * c - b * n, b * c + a * n], dim=-1).flatten(-2), x[..., rot:]], dim=-1)


def _angles(s):
    part = s["positions"].double()[:, None] * s["turns"][None, :]           # in 64 bits: positions are far
    a = (part - part.floor()) * (2 * math.pi)
    return (a.cos() * s["factor"]).float(), (a.sin() * s["factor"]).float()


def _plain_rotary(s):
    case = s["case"]
    cos, sin = _angles(s)
    if case["backward"]:
        sin = -sin
    return [_turned(s[x].float(), cos, sin, case["rot"], case["layout"]).to(s[x].dtype) for x in ("q", "k")]


def _plain_table(s):
    case = s["case"]
    P, off, cap, pages = case["page"], case["offset"], s["capacity"], s["ring"].numel()
    past, new, table = s["past"].long(), s["new"].long(), s["table"].long()
    head, count = s["ring_state"].long()
    R, W = table.shape
    have, gone = (past + P - 1) // P, new < 0
    more = torch.where(gone, 0, new)
    need = torch.where(gone, 0, (past + more + P - 1) // P - have)
    back = torch.where(gone, have, 0)
    cu, pu, bu = ((torch.cat([x.new_zeros(1), x.cumsum(0)])) for x in (more, need, back))
    status = torch.stack([(pu[-1] - count).clamp(min=0), (have + need > W).sum(), (cu[-1] - cap).clamp(min=0),
                          (count + bu[-1] - pages).clamp(min=0)])
    ok = (status == 0).all()
    lens = torch.where(ok, torch.where(gone, 0, past + more), past)
    state = torch.where(ok, torch.stack([(head + pu[-1]) % pages, count - pu[-1] + bu[-1]]), s["ring_state"].long())
    # pages given back go behind the ring's last
    at = (torch.arange(pages, device=table.device) - head - count) % pages
    giver = (torch.searchsorted(bu, at, right=True) - 1).clamp(max=R - 1)
    ring = torch.where(ok & (at < bu[-1]), table[giver, (at - bu[giver]).clamp(0, W - 1)], s["ring"].long())
    # and the ring's first go to the rows that need some
    j = torch.arange(W, device=table.device)[None, :]
    fresh = ok & (j >= have[:, None]) & (j < (have + need)[:, None])
    table = torch.where(fresh, s["ring"].long()[(head + pu[:-1, None] + j - have[:, None]) % pages], table)
    t = torch.arange(cap, device=table.device)
    r = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=R - 1)
    place = past[r] + t - cu[r]
    real = ok & (t < cu[-1])
    slots = torch.where(real, table[r, (place // P).clamp(max=W - 1)] * P + place % P, -1)
    positions = torch.where(real, place + off, 0)
    return [x.to(torch.int32) for x in (table, ring, state, lens, torch.where(ok, cu, 0), positions, slots, status)]


def _plain_append(s):
    case = s["case"]
    cos, sin = _angles(s)
    at = (s["slots"] >= 0).nonzero()[:, 0]
    slots = s["slots"].long()[at]
    q, k = (_turned(s[x].float(), cos, sin, case["rot"], case["layout"]).to(s[x].dtype) for x in ("q", "k"))
    s["q_out"][at] = q[at]
    s["k_pages"].view(-1, case["hkv"], case["d"])[slots] = k[at]
    s["v_pages"].view(-1, case["hkv"], case["d"])[slots] = s["v"][at]
    return s["q_out"], s["k_pages"], s["v_pages"]


def _plain_prefix(s):
    case = s["case"]
    T, Hq, Hkv, d = s["q"].shape[0], case["hq"], case["hkv"], case["d"]
    G, R, N, dev = Hq // Hkv, case["requests"], s["max_new"], s["q"].device
    cu = s["cu"].long() if s["cu"] is not None else torch.arange(R + 1, device=dev)
    q = s["q"].float() * s["scale"]
    # the prefix: one product for all requests
    rows = q.view(T, Hkv, G, d).transpose(0, 1).reshape(Hkv, T * G, d)
    s1 = rows @ s["prefix_k"].float().permute(1, 2, 0)                      # [Hkv, T G, L]
    # the suffixes: every request's pages, in front of N rows of queries
    S = s["max_suffix"]
    table = s["table"].long().clamp(min=0)
    k, v = (s[x].float()[table].view(R, S, Hkv, d).transpose(1, 2) for x in ("k_pages", "v_pages"))
    n, length = cu[1:] - cu[:-1], s["lens"].long()
    i, j = torch.arange(N, device=dev), torch.arange(S, device=dev)
    token = (cu[:-1, None] + i[None, :]).clamp(max=T - 1)                   # [R, N]
    seen = j[None, None, :] <= (length - n)[:, None, None] + i[None, :, None]
    qs = q[token].view(R, N, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(R, Hkv, N * G, d)
    s2 = (qs @ k.transpose(2, 3)).view(R, Hkv, N, G, S)
    s2 = s2.masked_fill(~seen[:, None, :, None, :], float("-inf"))
    v = torch.where((j[None, :] < length[:, None])[:, None, :, None], v, 0.0)
    # both in the order of the tokens' rows
    t = torch.arange(T, device=dev)
    r = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=R - 1)
    m1 = s1.amax(dim=2).view(Hkv, T, G)
    m2 = s2.amax(dim=4)                                                     # [R, Hkv, N, G]
    place = (t - cu[r]).clamp(max=N - 1)
    m = torch.maximum(m1, m2[r, :, place].transpose(0, 1))                  # [Hkv, T, G]
    p1 = (s1 - m.view(Hkv, T * G, 1)).exp_()
    m_there = m[:, token].permute(1, 0, 2, 3)                               # [R, Hkv, N, G]
    p2 = (s2 - m_there[..., None]).exp_()
    o2 = (p2.view(R, Hkv, N * G, S) @ v).view(R, Hkv, N, G, d)
    total = p1.sum(dim=2).view(Hkv, T, G) + p2.sum(dim=4)[r, :, place].transpose(0, 1)
    o = (p1 @ s["prefix_v"].float().transpose(0, 1)).view(Hkv, T, G, d) + o2[r, :, place].transpose(0, 1)
    o = (o / total[..., None]).transpose(0, 1).reshape(T, Hq, d).to(s["q"].dtype)
    real = t < cu[-1]
    out = [torch.where(real[:, None, None], o, s["out"])]
    if s["lse"] is not None:
        lse = (m + total.log()).transpose(1, 2).reshape(Hq, T)
        out.append(torch.where(real[None, :], lse, s["lse"]))
    return out


def _own_rotary(s):
    if "call" not in s:
        from paper_2603_06274_amd import decode_binding as db
        case = s["case"]
        s["call"] = db.stem_rotary, db.RotaryShape.from_tensors(s["q"], s["k"], case["rot"], case["layout"], s["q_out"], s["k_out"])
    call, shape = s["call"]
    call(shape, s["q"], s["k"], s["positions"], s["turns"], s["factor"], s["q_out"], s["k_out"], s["case"]["backward"])
    return s["q_out"], s["k_out"]


def _own_table(s):
    if "call" not in s:
        from paper_2603_06274_amd import decode_binding as db
        case = s["case"]
        shape = db.TableShape(case["requests"], case["page"], s["ring"].numel(), s["table"].shape[1], s["capacity"], case["offset"])
        space = torch.empty(db.stem_block_table_workspace_bytes(shape), dtype=torch.uint8, device=s["table"].device)
        s["call"] = db.stem_block_table, shape, space
    call, shape, space = s["call"]
    call(shape, s["past"], s["new"], s["ring_state"], s["ring"], s["table"], s["lens"], s["ring_state_out"], s["cu"],
         s["positions"], s["slots"], s["status"], space)
    return s["table"], s["ring"], s["ring_state_out"], s["lens"], s["cu"], s["positions"], s["slots"], s["status"]


def _own_append(s):
    if "call" not in s:
        from paper_2603_06274_amd import decode_binding as db
        case = s["case"]
        s["call"] = (db.stem_rotary_append, db.RotaryShape.from_tensors(s["q"], s["k"], case["rot"], case["layout"], s["q_out"]),
                     db.PageShape.from_tensors(s["k_pages"], s["v_pages"]))
    call, shape, pages = s["call"]
    call(shape, pages, s["q"], s["k"], s["v"], s["positions"], s["slots"], s["turns"], s["factor"], s["q_out"],
         s["k_pages"], s["v_pages"])
    return s["q_out"], s["k_pages"], s["v_pages"]


def _own_prefix(s):
    if "call" not in s:
        from paper_2603_06274_amd import decode_binding as db
        pages = db.PageShape.from_tensors(s["k_pages"], s["v_pages"])
        shape = db.PrefixShape.from_tensors(s["q"], s["prefix_k"], pages, s["table"], s["max_new"], s["max_suffix"])
        space = torch.empty(db.stem_prefix_attn_workspace_bytes(shape), dtype=torch.uint8, device=s["q"].device)
        s["call"] = db.stem_prefix_attn, shape, space
    call, shape, space = s["call"]
    call(shape, s["q"], s["prefix_k"], s["prefix_v"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["cu"],
         s["scale"], s["out"], s["lse"], space)
    return [s["out"]] if s["lse"] is None else [s["out"], s["lse"]]


PLAIN = {"rotary": _plain_rotary, "table": _plain_table, "append": _plain_append, "prefix": _plain_prefix}
OWN = {"rotary": _own_rotary, "table": _own_table, "append": _own_append, "prefix": _own_prefix}


# --- the definitions, in 64 bits ------------------------------------------------------------------------

def _spun(x, positions, turns, factor, rot, layout, backward):
    """Each pair as a complex number, times factor e^(+-i angle)."""
    angle = 2 * math.pi * torch.remainder(positions.double()[:, None] * turns, 1.0)
    spin = torch.polar(torch.full_like(angle, factor), -angle if backward else angle)[:, None, :]
    y = x.double()
    first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    z = torch.complex(y[..., first], y[..., second]) * spin
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    if case["op"] == "table":
        return None                                                         # whole numbers all
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return [_spun(s[x], s["positions"], s["turns"], s["factor"], case["rot"], case["layout"], case["backward"]) for x in ("q", "k")]
    past, new = _lens(case)
    if case["op"] == "append":
        q, k = (_spun(s[x], s["positions"], s["turns"], s["factor"], case["rot"], case["layout"], False) for x in ("q", "k"))
        real = sum(new)
        q_out, k_pages, v_pages = s["q_out"].double(), s["k_pages"].double(), s["v_pages"].double()
        q_out[:real] = q[:real]
        page, at = s["slots"][:real].long() // case["page"], s["slots"][:real].long() % case["page"]
        k_pages[page, at], v_pages[page, at] = k[:real], s["v"][:real].double()
        return q_out, k_pages, v_pages
    T, P, G = _tokens(case), case["page"], case["hq"] // case["hkv"]
    pk, pv = (s[x].double().transpose(0, 1).contiguous() for x in ("prefix_k", "prefix_v"))
    out = s["out"].double()
    lse = s["lse"].double() if s["lse"] is not None else None
    t = 0
    for r, (p, n) in enumerate(zip(past, new)):
        mine = s["table"][r, :_pages(p + n, P)].long()
        k, v = (s[x][mine].double().flatten(0, 1)[:p + n].transpose(0, 1) for x in ("k_pages", "v_pages"))
        for i in range(n):
            q = s["q"][t].double().view(case["hkv"], G, case["d"])
            logits = torch.cat([q @ pk.transpose(1, 2), q @ k[:, :p + i + 1].transpose(1, 2)], dim=2) * s["scale"]
            z = torch.logsumexp(logits, dim=2)
            w = (logits - z[..., None]).exp()
            o = w[..., :case["prefix"]] @ pv + w[..., case["prefix"]:] @ v[:, :p + i + 1]
            out[t] = o.reshape(case["hq"], case["d"])
            if lse is not None:
                lse[:, t] = z.flatten()
            t += 1
    return [out] if lse is None else [out, lse]
