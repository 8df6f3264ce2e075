"""Plain references in 64 bits, on the CPU, of the operators in include/stem_decode.h, and the bounds that the GPU tests hold them to.

A rounding to a type is off by at most EPS[type] / 2 of the value, EPS = torch.finfo(type).eps; u = 2^-24 is that of fp32."""
import math

import torch

U = 2.0 ** -24
EPS = {t: torch.finfo(t).eps for t in (torch.bfloat16, torch.float16, torch.float32, torch.float64)}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0,
        torch.float64: 0.0}            # half the step of fp16's subnormals


def rotary_reference(x, positions, turns, factor, rot, layout, backward=False):
    """(y, bound) of x [T, H, d] (any type, taken to 64 bits).

    The kernel's c and s are off by at most 4 u f: the reduced angle is rounded once and multiplied by 2 pi (2 u of an angle below
    pi / 4: < 1.6 u), the polynomials end with at most 2 u of rounding, the factor rounds once more and is itself rounded to fp32 (1 u
    relative each).  So c and s: 6 u f.  Two products, a sum: 3 roundings of at most (|x1| + |x2|) f.  In all 9 u f (|x1| + |x2|), then the
    rounding to the type."""
    a = 2 * math.pi * torch.remainder(positions.double()[:, None] * turns, 1.0)
    c, s = factor * torch.cos(a)[:, None, :], factor * torch.sin(a)[:, None, :]
    if backward:
        s = -s
    x64 = x.double()
    lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    y, bound = x64.clone(), torch.zeros_like(x64)
    y[..., lo] = x64[..., lo] * c - x64[..., hi] * s
    y[..., hi] = x64[..., hi] * c + x64[..., lo] * s
    fp32 = 9 * U * abs(factor) * (x64[..., lo].abs() + x64[..., hi].abs())
    for part in (lo, hi):
        bound[..., part] = fp32 + EPS[x.dtype] / 2 * (y[..., part].abs() + fp32) + TINY[x.dtype]
    return y, bound                                    # behind the rotary part: exact


def table_step(P, W, N, cap, off, past, new, ring, state, table):
    """What stem_block_table says of one step, in Python numbers.  ring and table (lists) are changed in place."""
    R, most = len(past), W * P
    pages = lambda n: -(-n // P)
    head, count = state
    good = 0 <= head < N and 0 <= count <= N
    bad = sum(p < 0 or p + max(n, 0) > most for p, n in zip(past, new))
    fine = [(p, n) if not (p < 0 or p + max(n, 0) > most) else (0, 0) for p, n in zip(past, new)]
    need = [0 if n < 0 else pages(p + n) - pages(p) for p, n in fine]
    back = [pages(p) if n < 0 else 0 for p, n in fine]
    more = [max(n, 0) for _, n in fine]
    h, c = (head, count) if good else (0, 0)
    status = [max(sum(need) - c, 0), bad, max(sum(more) - cap, 0), max(c + sum(back) - N, 0) if good else 1]
    if any(status):
        return dict(status=status, lens=list(past), state=list(state), cu=[0] * (R + 1), positions=[0] * cap, slots=[-1] * cap)
    then = list(ring)
    taken = given = 0
    for r in range(R):
        for i in range(need[r]):
            table[r][pages(past[r]) + i] = then[(h + taken) % N]
            taken += 1
        for i in range(back[r]):
            ring[(h + c + given) % N] = table[r][i]
            given += 1
    lens, cu, positions, slots = [], [0], [], []
    for r in range(R):
        for i in range(more[r]):
            at = past[r] + i
            page = table[r][at // P]
            positions.append(off + at)
            slots.append(page * P + at % P if 0 <= page < N else -1)
        lens.append(0 if new[r] < 0 else past[r] + new[r])
        cu.append(cu[-1] + more[r])
    rest = cap - cu[-1]
    return dict(status=status, lens=lens, state=[(h + taken) % N, c - taken + given], cu=cu, positions=positions + [0] * rest,
                slots=slots + [-1] * rest)


def attention_rows(q, k, v, scale, dtype):
    """(o, bound, lse, lse bound) of rows q [H, d] over keys k [n, H, d], v [n, H, d], all in 64 bits.

    Scores: a product of two values is exact in fp32, d sums round (u each of the sum of magnitudes S so far); scale, log2(e), the
    reference and the exponential's own error add 4 u of |s| and 2 u: a weight is off by a relative e = (d + 4) u S scale + 4 u |s| + 4 u.
    The reference is up to 8 powers of two below the largest score, which changes none of this.  Weights, unrounded, sum up in fp32 (n u),
    are rounded to the type for the second product (eps / 2; in fp16 also by half a subnormal step, 2^-25 of a largest weight of
    at least 1 in the row), whose sums round (n u).  The parts' join adds 8 u.  With A = sum w |v|, D = e + n u + 8 u:
    |o' - o| <= (2 D + eps / 2) A + 2^-25 sum |v| (fp16) + eps / 2 |o| and lse is off by D plus u of itself and of the exponents."""
    n, d = k.shape[0], q.shape[-1]
    if n == 0:
        z = torch.zeros_like(q)
        return z, z.clone(), torch.full(q.shape[:1], -math.inf, dtype=torch.float64), torch.zeros(q.shape[0], dtype=torch.float64)
    kt, vt = k.transpose(0, 1), v.transpose(0, 1)      # [H, n, d]
    s = scale * (kt @ q[..., None])[..., 0]
    mags = scale * (kt.abs() @ q.abs()[..., None])[..., 0]
    lse = torch.logsumexp(s, dim=1)
    w = (s - lse[:, None]).exp()
    o = (w[:, None, :] @ vt)[:, 0]
    e = (d + 4) * U * mags.amax(dim=1) + 4 * U * (s.abs().amax(dim=1) + lse.abs()) + 4 * U
    D = e + n * U + 8 * U
    A = (w[:, None, :] @ vt.abs())[:, 0]
    eps = EPS[dtype]
    bound = (2 * D[:, None] + eps / 2 * (1 + D[:, None])) * A + eps / 2 * o.abs()
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25 * vt.abs().sum(dim=1) + TINY[dtype]
    return o, 1.01 * bound, lse, D + 4 * U * (lse.abs() + 1)


def gathered(pages, table_row, n, page_size):
    """Rows 0 .. n - 1 of a request's keys or values, in 64 bits, and which of them are there (their page is one of the cache's)."""
    at = torch.arange(n)
    page = table_row.long()[at // page_size]
    there = (page >= 0) & (page < pages.shape[0])
    return pages[page.clamp(0, pages.shape[0] - 1), at % page_size].double(), there


def prefix_reference(q, pk, pv, kp, vp, table, lens, cu, scale, max_new, max_suffix):
    """{token: (o, bound, lse, lse bound)} of the rows that stem_prefix_attn writes; everything on the CPU."""
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
            (K, there), (V, _) = gathered(kp, table[r], L, P), gathered(vp, table[r], L, P)
        for i in range(min(n, max_new)):
            sees = max(min(L - n + i + 1, L), 0) if L else 0
            k, v = K0, V0
            if sees:
                k, v = torch.cat([K0, K[:sees][there[:sees]]]), torch.cat([V0, V[:sees][there[:sees]]])
            k, v = (x.repeat_interleave(G, dim=1) for x in (k, v))
            out[first + i] = attention_rows(q[first + i].double(), k, v, scale, q.dtype)
    return out
