"""Plain references of the cache's operators (include/spear_kv.h), in 64 bits
and request by request, and the bounds that their results are held to."""
from __future__ import annotations

import math

import torch

TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}
U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # half a step, relative


def plain_pages(held, fresh, free, table, tokens, P):
    """Lists in, lists out: starts, lens, table, slots, positions, taken."""
    R, width = len(held), len(table[0]) if table else 0
    table = [list(row) for row in table]
    starts, lens, at, got = [0], [], 0, 0
    slots, positions = [-1] * tokens, [0] * tokens
    unserved, true_at, claimed = 0, 0, 0
    for r in range(R):
        h, f = held[r], fresh[r]
        rows = max(f, 0)
        begin = min(true_at, tokens)
        true_at += rows
        starts.append(min(true_at, tokens))
        ok = h >= 0 and f >= 0 and h + f < 2 ** 30 and true_at <= tokens and -(-(h + f) // P) <= width
        if ok:
            had, has = -(-h // P), -(-(h + f) // P)
            claimed += has - had
            ok = has == had or claimed <= len(free)
        if not ok:
            unserved += 1
            lens.append(0)
            continue
        lens.append(h + f)
        for j in range(had, has):
            table[r][j] = free[got]
            got += 1
        for i in range(f):
            p = h + i
            s = table[r][p // P] * P + p % P
            slots[begin + i] = s if table[r][p // P] >= 0 and s < 2 ** 31 else -1
            positions[begin + i] = p
    return starts, lens, table, slots, positions, [got, unserved]


def turned(x, positions, freqs, rot, interleaved, magnitude):
    """x [T][heads][D] in 64 bits; freqs: whole numbers of 2^-64 turns."""
    y = x.double().clone()
    if rot == 0:
        return y
    frac = torch.tensor([[(int(p) * f) % 2 ** 64 / 2 ** 64 for f in freqs] for p in positions], dtype=torch.float64)
    c, s = magnitude * torch.cos(2 * math.pi * frac), magnitude * torch.sin(2 * math.pi * frac)
    ia = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    ib = ia + 1 if interleaved else ia + rot // 2
    a, b = x.double()[:, :, ia], x.double()[:, :, ib]
    y[:, :, ia] = a * c[:, None] - b * s[:, None]
    y[:, :, ib] = b * c[:, None] + a * s[:, None]
    return y


def scale_for(top, codes):
    """Least power of two whose multiple by the largest code reaches top, 2^-100 at least."""
    e = -100
    while TOP[codes] * 2.0 ** e < top:
        e += 1
    return 2.0 ** e


def step_of(c, codes):
    """Distance between neighbouring codes at |c|."""
    if codes is torch.int8:
        return torch.ones_like(c)
    return torch.exp2(torch.clamp(torch.floor(torch.log2(c.abs() + 1e-300)), min=-6.0) - 3.0)


def nearest(c, codes):
    s = step_of(c, codes)
    return torch.round(c / s) * s


def top_code(scale, codes, act):
    reach = float(torch.finfo(act).max)
    return TOP[codes] if TOP[codes] * scale <= reach else (63.0 if codes is torch.int8 else 240.0)


def codes_of(t):
    """Codes of a cache tensor as 64-bit numbers, on the CPU."""
    return (t.cpu().double() if t.dtype is torch.int8 else t.cpu().float().double())


def check_written(before, after, x, slots, P, codes, act, slack):
    """K or V of a page pool, [pages][kv][P][D] (V turned round by the caller), before and after x
    [T][kv][D] (64 bits) went to `slots` in runs. slack [T][kv][D]: how far x itself may be off.
    before, after: (codes, scales) in 64 bits; what may differ is checked, the rest is equal."""
    (c0, s0), (c1, s1) = before, after
    want_c, want_s, free = c0.clone(), s0.clone(), torch.zeros_like(c0, dtype=torch.bool)
    pages = c0.shape[0]
    runs, t = [], 0
    while t < len(slots):
        if not 0 <= slots[t] < pages * P:
            t += 1
            continue
        n = 1
        while t + n < len(slots) and slots[t + n] == slots[t] + n and (slots[t] + n) % P:
            n += 1
        runs.append((t, n))
        t += n
    for t, n in runs:
        page, off = slots[t] // P, slots[t] % P
        for h in range(c0.shape[1]):
            v = x[t:t + n, h]
            size = torch.where(torch.isfinite(v), v.abs(), torch.zeros_like(v))
            lo = scale_for(float((size - slack[t:t + n, h]).clamp(min=0).max()), codes)
            hi = scale_for(float((size + slack[t:t + n, h]).max()), codes)
            got = float(s1[page, h])
            old = float(s0[page, h]) if off else 0.0
            assert max(old, lo) <= got <= max(old, hi), (page, h, got, lo, hi, old)
            want_s[page, h] = got
            if off and got > old:
                want_c[page, h, :off] = nearest(c0[page, h, :off] * (old / got), codes)
            most = top_code(got, codes, act)
            c = torch.where(torch.isnan(v), torch.zeros_like(v), v) / got
            c = c.clamp(-most, most)
            have = c1[page, h, off:off + n]
            near = nearest(c, codes)
            loose = torch.nan_to_num(slack[t:t + n, h]) / got
            fine = (have == near) | ((have - c).abs() <= 0.5 * torch.maximum(step_of(c, codes), step_of(have, codes)) + loose)
            fine &= (have == near) | (loose > 0)
            assert bool(fine.all()), (page, h, have[~fine][:4], c[~fine][:4])
            free[page, h, off:off + n] = True
    assert torch.equal(torch.where(free, c1, want_c), c1), "codes that no token went to"
    assert torch.equal(want_s, s1)


def plain_attention(q, k, v, starts, lens, heads, *, scale, softcap=0.0, slopes=None, window=0, prefix=None,
                    dead=None, max_new=None):
    """q [T][H][D]; k, v: for each request [len][kv][D] in 64 bits; dead: for each request a mask of
    tokens that no row sees. (out, bound): bound is how far an output of the act dtype may be."""
    T, H, D = q.shape
    u, act = U[q.dtype], q.dtype
    out, bound = torch.zeros((T, H, D), dtype=torch.float64), torch.zeros((T, H, D), dtype=torch.float64)
    for r in range(len(lens)):
        n, L = starts[r + 1] - starts[r], lens[r]
        m = min(n, max_new) if max_new else n
        if not m or not L:
            continue
        kv = k[r].shape[1]
        i = L - n + torch.arange(m)[:, None]
        j = torch.arange(L)[None, :]
        seen = (j <= i) & ((i - j < window) if window else True)
        if prefix is not None:
            seen = seen | (j < prefix[r])
        if dead is not None:
            seen = seen & ~dead[r][None, :L]
        for h in range(H):
            qs = q[starts[r]:starts[r] + m, h].double()
            kk, vv = k[r][:L, h * kv // H], v[r][:L, h * kv // H]
            kk, vv = (torch.where(seen.any(0)[:, None], z, torch.zeros_like(z)) for z in (kk, vv))
            s = scale * qs @ kk.T
            size = (abs(scale) * qs.abs() @ kk.abs().T)
            if softcap:
                s = softcap * torch.tanh(s / softcap)
            far = (i - j).abs().double()
            b = slopes[h] * far if slopes is not None else torch.zeros_like(far)
            s = (s - b).masked_fill(~seen, -math.inf)
            some = seen.any(1)
            p = torch.exp(s - torch.where(some, s.amax(1), torch.zeros(m).double())[:, None])
            p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
            o = p @ vv
            a = p @ vv.abs()
            # a score is off by its dot product and the few operations on it in fp32; its weight by as much,
            # relatively, and by its rounding; sums over L tokens by L steps of fp32 at most
            off = 2.0 ** -24 * ((D + 16) * size + 8 * (s.masked_fill(~seen, 0).abs() + b.abs()) + 16)
            po = p * off
            # The weights' roundings w (1 + d), |d| <= u: over the exact sum they put the output off by
            # sum p d v, at most u a. Over the sum of the rounded ones, as tiles have it, by
            # sum p (1 + d) v / sum p (1 + d) - o = sum p d (v - o) / (1 + sum p d), at most
            # u / (1 - u) sum p |v - o|; and sum p |v - o| <= a + |o|, and <= (sum p v^2 - o^2)^(1/2)
            # (sum p = 1, Cauchy and Schwarz).
            spread = torch.minimum(a + o.abs(), (p @ (vv * vv) - o * o).clamp(min=0).sqrt())
            weights = torch.maximum(u * a, u / (1 - u) * spread)
            e = weights + (po.sum(1, keepdim=True) + L * 2.0 ** -24) * a + po @ vv.abs() + u * o.abs()
            if act is torch.float16:
                # weights below 2^-14 of the largest are held to 2^-25; so is a value of v below 2^-14, which is
                # a code times any power of two and need not be one of fp16's multiples of 2^-24 (weights sum
                # to one: 2^-25 in all), and so is the output: 2^-25 once more
                e = e + 2.0 ** -25 * (L * vv.abs().amax() + 2)
            out[starts[r]:starts[r] + m, h], bound[starts[r]:starts[r] + m, h] = o, e + 1e-30
    return out, bound
