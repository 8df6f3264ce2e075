"""Normalised heads and drafted tokens, as timing cases: queries and keys normalised head by head and rotated by their
positions in one pass (with the gradients, and with the new keys and values written into their pages), and decoding steps
whose new tokens are a tree of drafts: its masks and positions, the attention over prefix, cache and tree, and what is kept of it.

A case's "op" names the operator:
  norm    heads normalised, scaled by weights and rotated; with "backward" the gradients of inputs and weights
  append  the same for a step's new tokens, keys and values written into their pages
  masks   which drafted tokens see which, and their positions, from every token's parent
  tree    attention of drafted tokens to a shared prefix, to their request's pages and to their ancestors
  accept  a step's keys and values written, the drafts that the model confirms found, their rows moved up, pages given back
Lengths of requests follow from the case alone ("lens_seed"), everything else from the seed.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


# --- cases ----------------------------------------------------------------------------------------------

def _norm(name, tokens, *, hq=32, hkv=8, d=128, rot=128, layout="half", theta=500000.0, start=0, seqs=1, dtype="bf16",
          weights="same", offset=0.0, backward=False):
    return _named(name, {"op": "norm", "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "rot": rot, "layout": layout,
                         "theta": theta, "start": start, "seqs": seqs, "dtype": dtype, "weights": weights,
                         "offset": offset, "backward": backward})


def _append(name, requests, *, hq=32, hkv=8, d=128, rot=128, layout="half", page=64, most_past=1024, most_new=1,
            padding=0, dtype="bf16", lens_seed=1):
    return _named(name, {"op": "append", "requests": requests, "hq": hq, "hkv": hkv, "d": d, "rot": rot, "layout": layout,
                         "page": page, "most_past": most_past, "most_new": most_new, "padding": padding, "dtype": dtype,
                         "theta": 500000.0, "weights": "same", "offset": 0.0, "lens_seed": lens_seed})


def _masks(name, requests, most_new, *, branch=4, most_past=4096, padding=0, lens_seed=1):
    return _named(name, {"op": "masks", "requests": requests, "most_new": most_new, "branch": branch,
                         "most_past": most_past, "padding": padding, "lens_seed": lens_seed})


def _tree(name, requests, most_new, *, prefix=0, most_past=1024, hq=32, hkv=8, d=128, page=64, branch=4, padding=0,
          lse=False, dtype="bf16", lens_seed=1):
    return _named(name, {"op": "tree", "requests": requests, "most_new": most_new, "prefix": prefix, "most_past": most_past,
                         "hq": hq, "hkv": hkv, "d": d, "page": page, "branch": branch, "padding": padding, "lse": lse,
                         "dtype": dtype, "lens_seed": lens_seed})


def _accept(name, requests, most_new, *, hkv=8, d=128, page=64, most_past=1024, branch=4, ids=64, padding=0, dtype="bf16",
            lens_seed=1):
    return _named(name, {"op": "accept", "requests": requests, "most_new": most_new, "hq": 0, "hkv": hkv, "d": d, "rot": d,
                         "layout": "half", "page": page, "most_past": most_past, "branch": branch, "ids": ids,
                         "padding": padding, "dtype": dtype, "theta": 500000.0, "weights": "same", "offset": 0.0,
                         "lens_seed": lens_seed})


def _named(name, case):
    return {"name": name, **case} if name else case


def listed():
    return [
        # One new token of each of 64 requests on its way into the cache: a decoding step, latency.
        _append("norm_append_decode", 64),
        # The headline layer's whole prompt before it is pre-filled.
        _norm("norm_128k", 131072),
        # Packed prompts of an odd total, half of each head rotated in neighbouring pairs, weights kept as what they
        # differ from one by, in fp16.
        _norm("norm_packed_part", 40961, hq=28, hkv=4, rot=64, layout="interleaved", theta=10000.0, seqs=7, dtype="fp16",
              weights="fp32", offset=1.0),
        # A long training sequence on its way back.
        _norm("norm_backward_32k", 32768, backward=True),
        # A small model's training batch of odd length, in fp32.
        _norm("norm_backward_fp32", 9001, hq=16, hkv=8, d=64, rot=64, seqs=3, dtype="fp32", backward=True),
        # Trees of a few drafts for every request of a step.
        _masks("masks_decode", 64, 16),
        # Wide trees on a busy server.
        _masks("masks_wide", 500, 256, branch=12, padding=77),
        # A handful of short chats on a small model: launches and latency.
        _tree("tree_small", 4, 8, most_past=700, hq=8, hkv=2, d=64, page=16),
        # Long chats without anything in common: as much arithmetic as memory traffic.
        _tree("tree_chats_32k", 16, 32, most_past=32768, lse=True),
        # Samples from the headline prompt, each with a tree of drafts; seven query heads per KV head, a padded batch,
        # fp16.
        _tree("tree_prefix_64k", 24, 12, prefix=65535, most_past=1200, hq=28, hkv=4, page=16, padding=5, dtype="fp16"),
        # What one step keeps of small trees.
        _accept("accept_decode", 16, 16),
        # The same on a busy server with small pages.
        _accept("accept_busy", 500, 64, page=16, branch=8, ids=32, padding=31),
    ]


HEADS = [(32, 8), (28, 4), (32, 8), (28, 4), (16, 8), (8, 1), (4, 4), (1, 1)]


def _between(rng, lo, hi):
    """A whole number, spread over the logarithm of the range."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    most["append"] = most["accept"]                     # prompts' new tokens, as many as a busy server's drafts
    while True:
        op = rng.choice(["norm", "norm", "append", "masks", "tree", "tree", "tree", "accept"])
        hq, hkv = rng.choice(HEADS)
        d = rng.choice([128, 128, 64, 256])
        seed = rng.randrange(1 << 20)
        page = rng.choice([16, 32, 64, 128])
        layout = rng.choice(["half", "interleaved"])
        rot = rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)])
        branch = rng.choice([1, 2, 4, 12, 64])
        padding = rng.choice([0, 0, rng.randint(1, 99)])
        if op == "norm":
            case = _norm("", _between(rng, 1, 131072), hq=hq, hkv=hkv, d=d, rot=rot, layout=layout,
                         theta=rng.choice([10000.0, 500000.0, 1000000.0]), start=rng.choice([0, rng.randrange(1 << 20)]),
                         seqs=rng.choice([1, 1, rng.randint(1, 9)]), dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                         weights=rng.choice(["same", "same", "fp32", "none"]), offset=rng.choice([0.0, 0.0, 1.0]),
                         backward=rng.random() < 0.5)
        elif op == "append":
            case = _append("", _between(rng, 1, 200), hq=hq, hkv=hkv, d=d, rot=rot, layout=layout, page=page,
                           most_past=_between(rng, 1, 2000), most_new=rng.choice([1, _between(rng, 1, 600)]),
                           padding=padding, dtype=rng.choice(["bf16", "bf16", "fp16"]), lens_seed=seed)
        elif op == "masks":
            case = _masks("", _between(rng, 1, 500), _between(rng, 1, 256), branch=branch,
                          most_past=_between(rng, 1, 32768), padding=padding, lens_seed=seed)
        elif op == "tree":
            case = _tree("", _between(rng, 1, 48), _between(rng, 1, 128), prefix=rng.choice([0, _between(rng, 1, 65535)]),
                         most_past=_between(rng, 1, 32768), hq=hq, hkv=hkv, d=d, page=page, branch=branch,
                         padding=min(padding, 9), lse=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "fp16"]),
                         lens_seed=seed)
            # the plain form's scores and its copies of the pages: a few GiB
            rows = case["requests"] * case["most_new"] * hq
            if rows * (case["prefix"] + case["most_past"]) > 1 << 29 or case["requests"] * case["most_past"] * hkv * d > 1 << 29:
                continue
        else:
            case = _accept("", _between(rng, 1, 500), _between(rng, 1, 128), hkv=hkv, d=d, page=page,
                           most_past=_between(rng, 1, 2000), branch=branch, ids=rng.choice([32, 64]), padding=padding,
                           dtype=rng.choice(["bf16", "bf16", "fp16"]), lens_seed=seed)
        if _cost(case) <= most[op]:
            return case


def _lens(case):
    """Tokens that each request has in its pages, and new ones of this step."""
    r = random.Random(case["lens_seed"])
    past = [r.randint(0, case["most_past"]) for _ in range(case["requests"])]
    new = [r.randint(1, case["most_new"]) if case["most_new"] > 1 else 1 for _ in range(case["requests"])]
    if case["most_new"] > 1:
        new[r.randrange(case["requests"])] = case["most_new"]
        if case["requests"] > 2:
            new[r.randrange(case["requests"])] = 0              # a request that waits this step
    return past, new


def _tokens(case):
    """Rows of the step's tensors: the new tokens, and what the batch is padded with."""
    return sum(_lens(case)[1]) + case["padding"]


def _pages(n, page):
    return -(-n // page)


def _words(n):
    return -(-n // 64)


def work(case):
    size = BYTES[case["dtype"]] if "dtype" in case else 4
    if case["op"] == "norm":
        values = case["tokens"] * (case["hq"] + case["hkv"]) * case["d"]
        moved, each = (3, 16) if case["backward"] else (2, 8)
        return {"bytes": moved * size * values + 4 * case["tokens"] + 2 * size * case["d"], "flops": each * values}
    past, new = _lens(case)
    tokens = sum(new)
    if case["op"] == "append":
        values = tokens * (case["hq"] + 2 * case["hkv"]) * case["d"]
        return {"bytes": 2 * size * values + 8 * tokens, "flops": 8 * values}
    if case["op"] == "masks":
        return {"bytes": tokens * (8 + 8 * _words(case["most_new"])) + 8 * case["requests"], "flops": 2 * tokens}
    if case["op"] == "accept":
        values = 2 * tokens * case["hkv"] * case["d"]
        return {"bytes": 2 * size * values + tokens * (16 + case["ids"] // 4) + 16 * case["requests"], "flops": 4 * values}
    keys = case["prefix"] + sum(p + n for p, n in zip(past, new))
    pairs = tokens * case["prefix"] + sum(n * (p + 1) for p, n in zip(past, new))
    return {"bytes": size * case["d"] * (2 * keys * case["hkv"] + 2 * tokens * case["hq"]) + 8 * tokens * _words(case["most_new"]),
            "flops": 4 * case["d"] * case["hq"] * pairs}


# --- inputs ---------------------------------------------------------------------------------------------

def _whole(values, dev):
    return torch.tensor(values, dtype=torch.int32, device=dev)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    s = {"op": case["op"], "case": case}

    def normal(*shape, scale=None):
        x = torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)
        return (x if scale is None else x * scale).to(TYPES[case["dtype"]])

    def uniform(n):
        return torch.rand(n, generator=g, device=dev, dtype=torch.float64)

    if "weights" in case:                               # what the norms and the rotation need
        d, rot = case["d"], case["rot"]
        s["turns"] = torch.tensor([case["theta"] ** (-2.0 * i / rot) / (2 * math.pi) for i in range(rot // 2)],
                                  dtype=torch.float64, device=dev)
        s["eps"], s["offset"] = 1e-6, case["offset"]
        s["qw"] = s["kw"] = None
        if case["weights"] != "none":
            kind = TYPES["fp32" if case["weights"] == "fp32" else case["dtype"]]
            s["qw"], s["kw"] = ((1.0 - case["offset"] + 0.2 * torch.randn(d, generator=g, device=dev)).to(kind) for _ in range(2))

    def rows(T, heads):
        # heads of different sizes, as projections have them
        return normal(T, heads, case["d"], scale=torch.exp(torch.randn(heads, 1, generator=g, device=dev))) if heads else None

    if case["op"] == "norm":
        T, n = case["tokens"], _pages(case["tokens"], case["seqs"])
        s["positions"] = (torch.arange(T, device=dev) % n + case["start"]).to(torch.int32)
        s["q"], s["k"] = rows(T, case["hq"]), rows(T, case["hkv"])
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        if case["backward"]:
            s["gq"], s["gk"] = normal(T, case["hq"], case["d"]), normal(T, case["hkv"], case["d"])
            s["gqw"], s["gkw"] = (torch.empty(case["d"], dtype=torch.float32, device=dev) for _ in range(2))
        return s

    past, new = _lens(case)
    R, N, T = case["requests"], max(max(new), 1), _tokens(case)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    real = cu[-1]
    s["max_new"] = N
    s["lens"], s["cu"] = _whole([p + n for p, n in zip(past, new)], dev), _whole(cu, dev)
    owner = torch.repeat_interleave(torch.arange(R, device=dev), torch.tensor(new, device=dev))
    index = torch.arange(real, device=dev) - s["cu"].long()[owner]          # of a token among its request's new ones
    if "branch" in case:
        # a token's parent is one of the `branch` tokens before it (1: a chain); the first has none
        back = (uniform(real) * index.clamp(max=case["branch"])).long()
        s["parents"] = torch.full((T,), -1, dtype=torch.int32, device=dev)
        s["parents"][:real] = torch.where(index > 0, index - 1 - back, -1).to(torch.int32)
        s["offset_of_positions"] = case.get("prefix", 0)
    if case["op"] == "masks":
        s["masks"] = torch.zeros(T, _words(N), dtype=torch.int64, device=dev)
        s["positions"] = torch.zeros(T, dtype=torch.int32, device=dev)
        s["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
        return s

    P = case["page"]
    need = [_pages(p + n, P) for p, n in zip(past, new)]
    most = max(need) + 3                                                    # entries of a table row
    pages = sum(need) + 5
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    first = torch.tensor(need, device=dev).cumsum(0) - torch.tensor(need, device=dev)
    at = torch.arange(most, device=dev)
    own_page = at[None, :] < torch.tensor(need, device=dev)[:, None]
    s["table"] = torch.where(own_page, order[(first[:, None] + at[None, :]).clamp(max=pages - 1)], -1).contiguous()
    s["k_pages"], s["v_pages"] = (normal(pages, P, case["hkv"], case["d"]) for _ in range(2))
    if case["op"] in ("append", "accept"):
        s["q"], s["k"], s["v"] = rows(T, case["hq"]), rows(T, case["hkv"]), normal(T, case["hkv"], case["d"])
        place = index + torch.tensor(past, device=dev)[owner]
        s["slots"] = torch.full((T,), -1, dtype=torch.int32, device=dev)
        s["slots"][:real] = (s["table"].long()[owner, place // P] * P + place % P).to(torch.int32)
        s["positions"] = torch.zeros(T, dtype=torch.int32, device=dev)
        s["positions"][:real] = place.to(torch.int32)
        s["q_out"] = normal(T, case["hq"], case["d"]) if case["hq"] else None    # what padding rows keep
        if case["op"] == "append":
            return s
        # drafts, and what the model says behind each: about three times in four one of the drafts that follow it
        ids = {32: torch.int32, 64: torch.int64}[case["ids"]]
        s["drafts"], s["targets"] = ((uniform(T) * 32000).to(ids) for _ in range(2))
        parent = s["parents"][:real].long()
        child = torch.where((uniform(real) < 0.75) & (parent >= 0), torch.arange(real, device=dev), -1)
        said = torch.full((T,), -1, dtype=torch.int64, device=dev)
        said.scatter_reduce_(0, (s["cu"].long()[owner] + parent.clamp(min=0)), child, "amax")
        s["targets"] = torch.where(said >= 0, s["drafts"][said.clamp(min=0)], s["targets"])
        s["ring"] = torch.full((pages,), -1, dtype=torch.int32, device=dev)
        head = int(torch.randint(pages, (1,), generator=g, device=dev))
        s["ring"][(torch.arange(5, device=dev) + head) % pages] = order[sum(need):]
        s["ring_state"] = _whole([head, 5], dev)
        s["ring_state_out"], s["lens_out"], s["accepted"], s["status"] = (
            torch.zeros(n, dtype=torch.int32, device=dev) for n in (2, R, R, 2))
        s["path"] = torch.full((T,), -1, dtype=torch.int32, device=dev)
        s["next"] = torch.zeros(R, dtype=ids, device=dev)
        return s

    # keys and queries with a common part, and first keys that every query looks at
    L, hkv, d, G = case["prefix"], case["hkv"], case["d"], case["hq"] // case["hkv"]
    common = normal(hkv, d)
    s["q"] = (normal(T, hkv, G, d) + 0.5 * common[:, None, :]).view(T, case["hq"], d)
    s["prefix_k"] = s["prefix_v"] = None
    if L:
        s["prefix_k"], s["prefix_v"] = normal(L, hkv, d), normal(L, hkv, d)
        s["prefix_k"][0] = 2.0 * common
    begins = s["table"][:, 0].long()
    s["k_pages"][begins[begins >= 0], 0] = 2.0 * common
    vis, _ = _ancestors(s["parents"].long(), s["cu"].long(), N)
    s["masks"] = _packed(vis)
    s["scale"] = d ** -0.5
    s["out"] = normal(T, case["hq"], d)                                     # what padding rows keep
    s["lse"] = torch.zeros(case["hq"], T, dtype=torch.float32, device=dev) if case["lse"] else None
    s["max_suffix"] = most * P
    return s


# --- one pass -------------------------------------------------------------------------------------------

def run(state):
    return (OWN if own else PLAIN)[state["op"]](state)


def _angles(s):
    part = s["positions"].double()[:, None] * s["turns"][None, :]           # in 64 bits: positions are far
    a = (part - part.floor()) * (2 * math.pi)
    return a.cos().float()[:, None, :], a.sin().float()[:, None, :]


def _turned(x, c, n, rot, layout):
    """x [T, H, d] in fp32, c and n (cosines and sines) [T, 1, rot / 2]."""
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * c - b * n, b * c + a * n, x[..., rot:]], dim=-1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * c - b * n, b * c + a * n], dim=-1).flatten(-2), x[..., rot:]], dim=-1)


def _full(weight, offset):
    return 1.0 if weight is None else weight.float() + offset


def _normed(s, x, weight):
    """x [T, H, d] normalised, scaled and turned."""
    x32 = x.float()
    n = x32 * torch.rsqrt((x32 * x32).mean(dim=-1, keepdim=True) + s["eps"]) * _full(weight, s["offset"])
    return _turned(n, *_angles(s), s["case"]["rot"], s["case"]["layout"]).to(x.dtype)


def _plain_norm(s):
    case = s["case"]
    if not case["backward"]:
        return [_normed(s, s["q"], s["qw"]), _normed(s, s["k"], s["kw"])]
    c, n = _angles(s)
    grads, weight_grads = [], []
    for x, gy, w in ((s["q"], s["gq"], s["qw"]), (s["k"], s["gk"], s["kw"])):
        x32 = x.float()
        r = torch.rsqrt((x32 * x32).mean(dim=-1, keepdim=True) + s["eps"])
        unit = x32 * r
        gn = _turned(gy.float(), c, -n, case["rot"], case["layout"])
        weight_grads.append((gn * unit).sum(dim=(0, 1), dtype=torch.float64).float())
        h = gn * _full(w, s["offset"])
        grads.append((r * (h - unit * (h * unit).mean(dim=-1, keepdim=True))).to(x.dtype))
    return grads if s["qw"] is None else grads + weight_grads


def _plain_append(s):
    at = (s["slots"] >= 0).nonzero()[:, 0]
    slots = s["slots"].long()[at]
    shape = s["k"].shape[1:]
    s["k_pages"].view(-1, *shape)[slots] = _normed(s, s["k"], s["kw"])[at]
    s["v_pages"].view(-1, *shape)[slots] = s["v"][at]
    if s["q"] is None:
        return s["k_pages"], s["v_pages"]
    s["q_out"][at] = _normed(s, s["q"], s["qw"])[at]
    return s["q_out"], s["k_pages"], s["v_pages"]


def _owners(cu, T):
    """Every row's request (the last for rows of nobody), and whether it is one's."""
    t = torch.arange(T, device=cu.device)
    return (torch.searchsorted(cu, t, right=True) - 1).clamp(max=cu.numel() - 2), t < cu[-1]


def _ancestors(parents, cu, N):
    """Which of its request's first N new tokens every token sees (its ancestors and itself), and its depth."""
    T, dev = parents.numel(), parents.device
    owner, real = _owners(cu, T)
    start = cu[owner]
    vis = torch.arange(N, device=dev)[None, :] == (torch.arange(T, device=dev) - start)[:, None]
    up = torch.where(parents >= 0, start + parents, -1)
    for _ in range(max(N - 1, 1).bit_length()):                             # twice as far each time
        has = up >= 0
        vis = vis | (vis[up.clamp(min=0)] & has[:, None])
        up = torch.where(has, up[up.clamp(min=0)], -1)
    vis = vis & real[:, None]
    return vis, vis.sum(dim=1) - 1


def _packed(bits):
    """Truth values [T, N] as the bits of 64-bit words."""
    T, N = bits.shape
    padded = torch.zeros(T, 64 * _words(N), dtype=torch.int64, device=bits.device)
    padded[:, :N] = bits
    return (padded.view(T, -1, 64) << torch.arange(64, device=bits.device)).sum(dim=2)


def _plain_masks(s):
    cu, T = s["cu"].long(), s["parents"].numel()
    vis, depth = _ancestors(s["parents"].long(), cu, s["max_new"])
    owner, real = _owners(cu, T)
    past = s["lens"].long() - (cu[1:] - cu[:-1])
    positions = torch.where(real, past[owner] + depth + s["offset_of_positions"], s["positions"].long())
    return torch.where(real[:, None], _packed(vis), s["masks"]), positions.to(torch.int32)


def _plain_tree(s):
    case = s["case"]
    T, Hq, Hkv, d = s["q"].shape[0], case["hq"], case["hkv"], case["d"]
    G, R, N, S, dev = Hq // Hkv, case["requests"], s["max_new"], s["max_suffix"], s["q"].device
    cu, length = s["cu"].long(), s["lens"].long()
    n = cu[1:] - cu[:-1]
    q = s["q"].float() * s["scale"]
    # every request's pages, in front of N rows of queries
    k, v = (s[x].float()[s["table"].long().clamp(min=0)].view(R, S, Hkv, d).transpose(1, 2) for x in ("k_pages", "v_pages"))
    token = (cu[:-1, None] + torch.arange(N, device=dev)[None, :]).clamp(max=T - 1)     # [R, N]
    j = torch.arange(S, device=dev)
    behind = j[None, :] - (length - n)[:, None]                             # a key's number among the new ones
    bit = behind.clamp(0, N - 1)[:, None, :].expand(R, N, S)
    masks = (s["masks"][token][..., None] >> torch.arange(64, device=dev)).flatten(2) & 1      # [R, N, 64 words]
    seen = (behind < 0)[:, None, :] | ((behind < n[:, None])[:, None, :] & (masks.gather(2, bit) != 0))
    qs = q[token].view(R, N, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(R, Hkv, N * G, d)
    s2 = (qs @ k.transpose(2, 3)).view(R, Hkv, N, G, S)
    s2 = s2.masked_fill(~seen[:, None, :, None, :], float("-inf"))
    v = torch.where((j[None, :] < length[:, None])[:, None, :, None], v, 0.0)
    t = torch.arange(T, device=dev)
    owner, real = _owners(cu, T)
    place = (t - cu[owner]).clamp(max=N - 1)
    m = s2.amax(dim=4)                                                      # [R, Hkv, N, G]
    if case["prefix"]:                                                      # one product for all requests
        rows = q.view(T, Hkv, G, d).transpose(0, 1).reshape(Hkv, T * G, d)
        s1 = rows @ s["prefix_k"].float().permute(1, 2, 0)                  # [Hkv, T G, L]
        m1 = s1.amax(dim=2).view(Hkv, T, G)
        m_row = torch.maximum(m1, m[owner, :, place].transpose(0, 1))       # [Hkv, T, G]
        m = m_row[:, token].permute(1, 0, 2, 3)
    p2 = (s2 - m[..., None]).exp_()
    o = ((p2.view(R, Hkv, N * G, S) @ v).view(R, Hkv, N, G, d))[owner, :, place].transpose(0, 1)
    total, m = p2.sum(dim=4)[owner, :, place].transpose(0, 1), m[owner, :, place].transpose(0, 1)   # [Hkv, T, G]
    if case["prefix"]:
        p1 = (s1 - m_row.view(Hkv, T * G, 1)).exp_()
        m = m_row
        total = total + p1.sum(dim=2).view(Hkv, T, G)
        o = o + (p1 @ s["prefix_v"].float().transpose(0, 1)).view(Hkv, T, G, d)
    o = (o / total[..., None]).transpose(0, 1).reshape(T, Hq, d).to(s["q"].dtype)
    out = [torch.where(real[:, None, None], o, s["out"])]
    if s["lse"] is not None:
        lse = (m + total.log()).transpose(1, 2).reshape(Hq, T)
        out.append(torch.where(real[None, :], lse, s["lse"]))
    return out


def _plain_accept(s):
    _plain_append(s)
    case, dev = s["case"], s["cu"].device
    P, R, T, N, pages = case["page"], case["requests"], s["parents"].numel(), s["max_new"], s["ring"].numel()
    cu, length, parents = s["cu"].long(), s["lens"].long(), s["parents"].long()
    n = cu[1:] - cu[:-1]
    owner, real = _owners(cu, T)
    t = torch.arange(T, device=dev)
    up = cu[owner] + parents.clamp(min=0)
    follows = real & (parents >= 0) & (s["drafts"] == s["targets"][up])
    after = torch.full((T,), T, device=dev).scatter_reduce(0, up, torch.where(follows, t, T), "amin")
    after = torch.cat([after, after.new_full((1,), T)])
    here = torch.where(n > 0, cu[:-1], T)                                   # [R], T: the walk has ended
    last, accepted = here, torch.zeros_like(here)
    path = torch.cat([s["path"].long().new_full((T,), -1), t.new_zeros(1)])
    for _ in range(N):
        on = here < T
        path[torch.where(on, cu[:-1] + accepted, T)] = torch.where(on, here - cu[:-1], 0)
        accepted = accepted + on
        last = torch.where(on, here, last)
        here = torch.where(on, after[here], T)
    path = torch.where(real, path[:T], s["path"].long())
    following = torch.where(n > 0, s["targets"].long()[last.clamp(max=T - 1)], -1)
    lens = length - n + accepted
    # rows of accepted drafts move up behind those before them
    rows = (real & (path >= 0)).nonzero()[:, 0]
    to, of = s["slots"].long()[rows], s["slots"].long()[(cu[owner] + path.clamp(min=0))[rows]]
    for x in ("k_pages", "v_pages"):
        flat = s[x].view(-1, case["hkv"], case["d"])
        flat[to] = flat[of]
    # pages behind the last kept token go behind the ring's last entry
    keep, had = (lens + P - 1) // P, (length + P - 1) // P
    before = torch.cat([keep.new_zeros(1), (had - keep).cumsum(0)])
    head, count = s["ring_state"].long()
    at = (torch.arange(pages, device=dev) - head - count) % pages
    giver = (torch.searchsorted(before, at, right=True) - 1).clamp(max=R - 1)
    entry = (keep[giver] + at - before[giver]).clamp(0, s["table"].shape[1] - 1)
    ring = torch.where(at < before[-1], s["table"].long()[giver, entry], s["ring"].long())
    state = torch.stack([head, count + before[-1]])
    return ([x.to(torch.int32) for x in (accepted, path, lens, ring, state)] +
            [following.to(s["next"].dtype), s["k_pages"], s["v_pages"]])


def _norm_call(s):
    """The prepared shapes of a call that normalises: what a program makes once."""
    from paper_2603_06274_amd import decode_binding as db
    from paper_2603_06274_amd import norm_binding as nb
    case = s["case"]
    return nb, db, nb.HeadNorm(s["qw"], s["kw"], s["eps"], s["offset"]), db.RotaryShape.from_tensors(
        s["q"], s["k"], case["rot"], case["layout"], s["q_out"], s.get("k_out"))


def _own_norm(s):
    if "call" not in s:
        nb, _, norm, shape = _norm_call(s)
        space = None
        if s["case"]["backward"]:
            space = torch.empty(nb.stem_norm_rotary_backward_workspace_bytes(shape), dtype=torch.uint8, device=s["q"].device)
        s["call"] = nb, norm, shape, space
    nb, norm, shape, space = s["call"]
    if not s["case"]["backward"]:
        nb.stem_norm_rotary(shape, norm, s["q"], s["k"], s["positions"], s["turns"], 1.0, s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    has = s["qw"] is not None
    nb.stem_norm_rotary_backward(shape, norm, s["q"], s["k"], s["positions"], s["turns"], 1.0, s["gq"], s["gk"], s["q_out"], s["k_out"],
                                 s["gqw"] if has else None, s["gkw"] if has else None, space)
    return (s["q_out"], s["k_out"], s["gqw"], s["gkw"]) if has else (s["q_out"], s["k_out"])


def _own_append(s):
    if "call" not in s:
        nb, db, norm, shape = _norm_call(s)
        s["call"] = nb, norm, shape, db.PageShape.from_tensors(s["k_pages"], s["v_pages"])
    nb, norm, shape, pages = s["call"]
    nb.stem_norm_rotary_append(shape, norm, pages, s["q"], s["k"], s["v"], s["positions"], s["slots"], s["turns"], 1.0, s["q_out"],
                               s["k_pages"], s["v_pages"])
    return (s["k_pages"], s["v_pages"]) if s["q"] is None else (s["q_out"], s["k_pages"], s["v_pages"])


def _own_masks(s):
    if "call" not in s:
        from paper_2603_06274_amd import tree_binding as tb
        s["call"] = tb, tb.TreeShape(s["case"]["requests"], s["parents"].numel(), s["max_new"], s["offset_of_positions"])
    tb, shape = s["call"]
    tb.stem_tree_masks(shape, s["parents"], s["lens"], s["cu"], s["positions"], s["masks"], s["status"])
    return s["masks"], s["positions"]


def _own_tree(s):
    if "call" not in s:
        from paper_2603_06274_amd import decode_binding as db
        from paper_2603_06274_amd import tree_binding as tb
        pages = db.PageShape.from_tensors(s["k_pages"], s["v_pages"])
        shape = db.PrefixShape.from_tensors(s["q"], s["prefix_k"], pages, s["table"], s["max_new"], s["max_suffix"])
        space = torch.empty(tb.stem_tree_attn_workspace_bytes(shape), dtype=torch.uint8, device=s["q"].device)
        s["call"] = tb, shape, space
    tb, shape, space = s["call"]
    tb.stem_tree_attn(shape, s["q"], s["prefix_k"], s["prefix_v"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["cu"],
                      s["masks"], s["scale"], s["out"], s["lse"], space)
    return [s["out"]] if s["lse"] is None else [s["out"], s["lse"]]


def _own_accept(s):
    if "call" not in s:
        from paper_2603_06274_amd import tree_binding as tb
        nb, db, norm, shape = _norm_call(s)
        case = s["case"]
        walk = tb.AcceptShape(case["requests"], s["parents"].numel(), s["max_new"], case["page"], s["ring"].numel(), s["table"].shape[1])
        space = torch.empty(tb.stem_tree_accept_workspace_bytes(walk), dtype=torch.uint8, device=s["table"].device)
        s["call"] = nb, tb, norm, shape, db.PageShape.from_tensors(s["k_pages"], s["v_pages"]), walk, space
    nb, tb, norm, shape, pages, walk, space = s["call"]
    nb.stem_norm_rotary_append(shape, norm, pages, None, s["k"], s["v"], s["positions"], s["slots"], s["turns"], 1.0, None,
                               s["k_pages"], s["v_pages"])
    tb.stem_tree_accept(walk, s["parents"], s["drafts"], s["targets"], s["cu"], s["lens"], s["ring_state"], s["ring"], s["table"],
                        s["lens_out"], s["ring_state_out"], s["accepted"], s["path"], s["next"], s["status"], space)
    tb.stem_tree_commit(walk, pages, s["path"], s["slots"], s["cu"], s["k_pages"], s["v_pages"])
    return s["accepted"], s["path"], s["lens_out"], s["ring"], s["ring_state_out"], s["next"], s["k_pages"], s["v_pages"]


PLAIN = {"norm": _plain_norm, "append": _plain_append, "masks": _plain_masks, "tree": _plain_tree, "accept": _plain_accept}
OWN = {"norm": _own_norm, "append": _own_append, "masks": _own_masks, "tree": _own_tree, "accept": _own_accept}


# --- the definitions, in 64 bits ------------------------------------------------------------------------

def _spun(x, weight, s):
    """x, in 64 bits, divided by its root mean square, times its weights, each pair times e^(i angle) as a complex number."""
    rot, layout = s["case"]["rot"], s["case"]["layout"]
    y = x / (x.square().sum(dim=-1, keepdim=True) / x.shape[-1] + s["eps"]).sqrt()
    if weight is not None:
        y = y * (weight + s["offset"])
    angle = 2 * math.pi * torch.remainder(s["positions"].double()[:, None] * s["turns"], 1.0)
    first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.ones_like(angle), angle)[:, None, :]
    out = y.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _wide(w):
    return None if w is None else w.double()


def exact(case, seed):
    if case["op"] == "masks":
        return None                                                         # whole numbers all
    s = prepare(case, seed)
    if case["op"] == "norm":
        if not case["backward"]:
            return [_spun(s[x].double(), _wide(s[x + "w"]), s) for x in ("q", "k")]
        grads, weight_grads = [], []
        for x in ("q", "k"):
            leaf, w = s[x].double().requires_grad_(), _wide(s[x + "w"])
            leaves = [leaf] if w is None else [leaf, w.requires_grad_()]
            g = torch.autograd.grad(_spun(leaf, w, s), leaves, s["g" + x].double())
            grads.append(g[0])
            weight_grads += g[1:]
        return grads + weight_grads
    past, new = _lens(case)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    P = case["page"]
    if case["op"] in ("append", "accept"):
        real, k_pages, v_pages = cu[-1], s["k_pages"].double(), s["v_pages"].double()
        page, at = s["slots"][:real].long() // P, s["slots"][:real].long() % P
        k_pages[page, at], v_pages[page, at] = _spun(s["k"].double(), _wide(s["kw"]), s)[:real], s["v"][:real].double()
        if case["op"] == "append":
            q_out = s["q_out"].double()
            q_out[:real] = _spun(s["q"].double(), _wide(s["qw"]), s)[:real]
            return q_out, k_pages, v_pages
        parents, drafts, targets = (s[x].tolist() for x in ("parents", "drafts", "targets"))
        to, of = [], []
        for first, n in zip(cu, new):
            here, k = 0, 0
            while n:
                to.append(first + k)
                of.append(first + here)
                k += 1
                here = next((c for c in range(here + 1, n) if parents[first + c] == here and
                             drafts[first + c] == targets[first + here]), None)
                if here is None:
                    break
        to, of = torch.tensor(to, device=page.device), torch.tensor(of, device=page.device)
        for x in (k_pages, v_pages):
            x[page[to], at[to]] = x[page[of], at[of]]
        return None, None, None, None, None, None, k_pages, v_pages
    hkv, G, d = case["hkv"], case["hq"] // case["hkv"], case["d"]
    out = s["out"].double()
    lse = s["lse"].double() if s["lse"] is not None else None
    parents = s["parents"].tolist()
    prefix = [s[x].double().transpose(0, 1) for x in ("prefix_k", "prefix_v")] if case["prefix"] else None
    for r, (p, n) in enumerate(zip(past, new)):
        if n == 0:
            continue
        rows = slice(cu[r], cu[r] + n)
        mine = s["table"][r, :_pages(p + n, P)].long()
        k, v = (s[x][mine].double().flatten(0, 1)[:p + n].transpose(0, 1) for x in ("k_pages", "v_pages"))
        if prefix:
            k, v = torch.cat([prefix[0], k], dim=1), torch.cat([prefix[1], v], dim=1)
        sees = torch.zeros(n, n, dtype=torch.bool)
        for i in range(n):
            up = parents[cu[r] + i]
            if up >= 0:
                sees[i] = sees[up]
            sees[i, i] = True
        q = s["q"][rows].double().view(n, hkv, G, d).permute(1, 2, 0, 3)    # [hkv, G, n, d]
        logits = (q.reshape(hkv, G * n, d) @ k.transpose(1, 2).contiguous()).view(hkv, G, n, -1) * s["scale"]
        logits[..., -n:].masked_fill_(~sees.to(logits.device), float("-inf"))
        z = torch.logsumexp(logits, dim=3)
        w = (logits - z[..., None]).exp().view(hkv, G * n, -1)
        out[rows] = (w @ v.contiguous()).view(hkv, G, n, d).permute(2, 0, 1, 3).reshape(n, case["hq"], d)
        if lse is not None:
            lse[:, rows] = z.reshape(case["hq"], n)
    return [out] if lse is None else [out, lse]
