"""Plain references, on the CPU, of the operators in include/stem_tree.h."""
import torch

import decode_util as du


def ancestors(parents, n):
    """For each of a request's n new tokens the set of those that it sees, and its depth; parents that are none count as -1."""
    sees, depth = [], []
    for i in range(n):
        p = parents[i]
        p = p if 0 <= p < i else -1
        sees.append((sees[p] if p >= 0 else set()) | {i})
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return sees, depth


def words(sees, count):
    """A set of numbers as `count` signed 64-bit words."""
    out = []
    for w in range(count):
        x = sum(1 << (j - 64 * w) for j in sees if 64 * w <= j < 64 * w + 64)
        out.append(x - (1 << 64) if x >> 63 else x)
    return out


def random_parents(rng, n, branch):
    return [-1 if i == 0 else i - 1 - rng.randrange(min(i, branch)) for i in range(n)]


def attention(q, pk, pv, kp, vp, table, lens, cu, masks, scale, max_new, max_suffix):
    """{token: (o, bound, lse, lse bound)} of the rows that stem_tree_attn writes; everything on the CPU, masks int64 [T, words]."""
    T, Hq, d = q.shape
    Hkv = pk.shape[1] if pk is not None else kp.shape[2]
    G, out = Hq // Hkv, {}
    empty = torch.zeros(0, Hkv, d, dtype=torch.float64)
    K0, V0 = (x.double() if x is not None else empty for x in (pk, pv))
    for r in range(len(cu) - 1):
        first = min(max(cu[r], 0), T)
        n = max(min(cu[r + 1], T) - first, 0)
        L = min(max(int(lens[r]), 0), max_suffix) if max_suffix else 0
        if L:
            P = kp.shape[1]
            (K, there), (V, _) = du.gathered(kp, table[r], L, P), du.gathered(vp, table[r], L, P)
        for i in range(min(n, max_new)):
            k, v = K0, V0
            if L:
                j = torch.arange(L) - (L - n)          # a key's number among the new tokens
                row = masks[first + i]
                bits = (row[(j // 64).clamp(0, len(row) - 1)] >> (j % 64)) & 1
                seen = there & ((j < 0) | ((bits != 0) & (j < 64 * len(row))))
                k, v = torch.cat([K0, K[seen]]), torch.cat([V0, V[seen]])
            k, v = (x.repeat_interleave(G, dim=1) for x in (k, v))
            out[first + i] = du.attention_rows(q[first + i].double(), k, v, scale, q.dtype)
    return out


def walk(parents, drafts, targets, n):
    """(path, next) of a request's n new tokens."""
    if n == 0:
        return [], -1
    path = [0]
    while True:
        here = path[-1]
        follow = [c for c in range(here + 1, n) if parents[c] == here and drafts[c] == targets[here]]
        if not follow:
            return path, targets[here]
        path.append(follow[0])


def accept(P, W, N, max_new, parents, drafts, targets, cu, lens, ring, state, table):
    """What stem_tree_accept says, in Python numbers.  ring (a list) is changed in place."""
    R, T = len(lens), len(parents)
    pages = lambda n: -(-n // P)
    head, count = state
    good = 0 <= head < N and 0 <= count <= N
    spans = []
    for r in range(R):
        first = min(max(cu[r], 0), T)
        spans.append((first, max(min(cu[r + 1], T) - first, 0)))
    bad = sum(n > max_new or lens[r] < n or lens[r] > W * P for r, (_, n) in enumerate(spans))
    walks = [walk(parents[f:f + n], drafts[f:f + n], targets[f:f + n], n) for f, n in spans]
    left = [lens[r] - n + len(walks[r][0]) for r, (_, n) in enumerate(spans)]
    back = [e for r in range(R) for e in range(pages(left[r]), pages(lens[r]))] if not bad else []
    no_room = max((count if good else 0) + len(back) - N, 0) if good else 1
    status = [bad, no_room]
    path = {}
    if any(status):
        for f, n in spans:
            path.update({f + i: -1 for i in range(n)})
        return dict(status=status, lens=list(lens), state=list(state), accepted=[0] * R, next=[-1] * R, path=path)
    given = 0
    for r, (f, n) in enumerate(spans):
        path.update({f + i: walks[r][0][i] if i < len(walks[r][0]) else -1 for i in range(n)})
        for e in range(pages(left[r]), pages(lens[r])):
            ring[(head + count + given) % N] = table[r][e]
            given += 1
    return dict(status=status, lens=left, state=[head, count + given], accepted=[len(w[0]) for w in walks], next=[w[1] for w in walks],
                path=path)
