"""What is timed of attention over a cache held in 8 bits, beside the 4-bit
linear layer that makes its queries, keys and values.

Kinds of case:

* "pages": block tables, slot maps and positions of a step, from the requests'
  lengths: each request's new pages taken from a list of free ones in order,
  and where in the cache every new token goes.
* "append": rotary positions on new queries and keys, and the new keys and
  values written to the cache in 8 bits, with one scale (a power of two) for
  each page of tokens and head; what was in a page before is brought to its new
  scale. Read back, every token of the pages that were written, as values.
* "attend": attention of the new tokens' queries over the cache, causal, of
  requests of unlike lengths; scores capped by a tanh, biased by distance,
  inside a window, with a prefix that every token sees.
* "step": all of them as one decoding step makes them.

Pages hold K as [page][head][token][feature] and V as [page][head][feature]
[token]. Head counts and widths are those of the Llama-3.2-1B, Llama-3-8B and
Llama-2-70B layers that this repository serves, one of eight tensor-parallel
shards, and generic ones. Queries, keys and values are N(0, 1), keys with some
features ten times as large.
"""
import math
import random

import torch

own = False

_DT = {"f16": torch.float16, "bf16": torch.bfloat16}
_CODE = {"f16": 0, "bf16": 1}
_HELD = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
_TOP = {"int8": 127.0, "e4m3": 448.0}
_LOW, _HIGH, _CONTEXT = 1.0, 4.0, 8192   # of the scaled rotary frequencies
_BASE = 500000.0


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _pages(R, new, most, *, P=64, short=0, pad=0, mix=1, name=None):
    c = dict(kind="pages", R=R, new=new, most=most, P=P, short=short, pad=pad, mix=mix)
    return dict(c, name=name) if name else c


def _append(R, new, most, heads, kv, D, *, P=64, fmt="int8", dtype="f16", rot=0, inter=False,
            factor=1.0, mix=1, name=None):
    c = dict(kind="append", R=R, new=new, most=most, heads=heads, kv=kv, D=D, P=P, fmt=fmt,
             dtype=dtype, rot=rot or D, inter=inter, factor=factor, mix=mix)
    return dict(c, name=name) if name else c


def _attend(R, new, least, most, heads, kv, D, *, single=0, P=64, fmt="int8", dtype="f16", cap=0.0,
            slopes=False, window=0, prefix=0, mix=1, name=None):
    c = dict(kind="attend", R=R, new=new, least=least, most=most, heads=heads, kv=kv, D=D, single=single,
             P=P, fmt=fmt, dtype=dtype, cap=cap, slopes=slopes, window=window, prefix=prefix, mix=mix)
    return dict(c, name=name) if name else c


def _step(R, least, most, heads, kv, D, *, P=64, fmt="int8", dtype="f16", mix=1, name=None):
    c = dict(kind="step", R=R, new=1, least=least, most=most, heads=heads, kv=kv, D=D, single=R, P=P,
             fmt=fmt, dtype=dtype, cap=0.0, slopes=False, window=0, prefix=0, rot=D, inter=False,
             factor=8.0, mix=mix)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a single request decoding: nothing but latency
        _pages(1, 1, 2000, P=16, name="pages, 1 request"),
        # a large serving batch, prompts among decoding requests, nine pages too few
        _pages(384, 64, 20000, P=32, short=9, pad=100, mix=3, name="pages, 384 requests"),
        # one token of the 8B model
        _append(1, 1, 3000, 32, 8, 128, P=16, name="append, 1 token"),
        # prompts of seven requests, rotary positions on part of the head, pairs side by side
        _append(7, 300, 5000, 12, 3, 64, P=32, fmt="e4m3", dtype="bf16", rot=32, inter=True, mix=2,
                name="append, 7 prompts, part of the head"),
        # a long prompt on the headline model, positions far out and scaled
        _append(1, 4096, 120000, 64, 8, 128, P=64, dtype="bf16", factor=8.0, name="append, 4096 tokens"),
        # one request on the small model, a short context
        _attend(1, 1, 500, 500, 32, 8, 64, single=1, P=16, name="1b, 1 request, 500 tokens"),
        # a decode batch of unlike lengths on the 8B model
        _attend(64, 1, 16, 8192, 32, 8, 128, single=64, P=32, fmt="e4m3", dtype="bf16", mix=4,
                name="8b, 64 requests"),
        # one long conversation on the headline model
        _attend(1, 1, 131000, 131000, 64, 8, 128, single=1, dtype="bf16", name="70b, 1 request, 131000 tokens"),
        # capped scores, a window, a bias by distance and a prefix; heads and lengths of no particular size
        _attend(13, 37, 1, 3000, 15, 5, 128, single=6, P=16, cap=30.0, slopes=True, window=1000,
                prefix=50, mix=5, name="13 requests, capped, window"),
        # a chunk of a long prompt beside decoding requests, a shard of the headline model
        _attend(9, 512, 5000, 8700, 8, 1, 128, single=8, fmt="e4m3", dtype="bf16", mix=6,
                name="70b/8, chunk of 512 and 8 requests"),
        # a long prompt on the headline model
        _attend(1, 4096, 4096, 4096, 64, 8, 128, name="70b, prompt of 4096"),
        # a decoding step of 24 requests on the 8B model, everything of it
        _step(24, 100, 6000, 32, 8, 128, fmt="e4m3", mix=7, name="8b, step of 24 requests"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("pages", "append", "append", "attend", "attend", "attend", "step"))
    mix, P = rng.randrange(1, 1 << 30), rng.choice((16, 32, 64, 128))
    if kind == "pages":
        return _pages(_log_uniform(rng, 1, 512), _log_uniform(rng, 1, 128), _log_uniform(rng, 200, 30000), P=P,
                      short=rng.choice((0, 0, 0, 2, 11)), pad=rng.choice((0, 0, 5, 64)), mix=mix)
    D, g, kv = rng.choice((64, 128)), rng.choice((1, 2, 3, 4, 7, 8)), rng.choice((1, 2, 3, 4, 8))
    opt = dict(P=P, fmt=rng.choice(("int8", "e4m3")), dtype=rng.choice(("f16", "bf16")), mix=mix)
    if kind == "append":
        R = _log_uniform(rng, 1, 64)
        new = 1 if rng.random() < 0.3 else _log_uniform(rng, 1, max(1, 4096 // R))
        return _append(R, new, new + _log_uniform(rng, 1, 200000), g * kv, kv, D,
                       rot=rng.choice((D, D, D // 2, D // 4, 6)), inter=rng.random() < 0.5,
                       factor=rng.choice((1.0, 8.0)), **opt)
    if kind == "step" or rng.random() < 0.5:
        R = _log_uniform(rng, 1, 64)
        most = min(131000, _log_uniform(rng, 8, 400000 // R))
        least = rng.choice((1, most, max(1, most // 20)))
        if kind == "step":
            return _step(R, least, most, g * kv, kv, D, **opt)
        return _attend(R, 1, least, most, g * kv, kv, D, single=R, **_options(rng, most), **opt)
    R = _log_uniform(rng, 1, 12)
    new = _log_uniform(rng, 2, 2000)
    # the scores of all requests, padded to the longest, stay under the largest listed case's
    most = max(new, min(16000, _log_uniform(rng, new, max(new + 1, 500_000_000 // (R * new * g * kv)))))
    R = max(1, min(R, 500_000_000 // (most * new * g * kv)))
    return _attend(R, new, rng.choice((1, max(1, most // 3), most)), most, g * kv, kv, D,
                   single=rng.choice((0, 0, R // 2)), **_options(rng, most), **opt)


def _options(rng, most):
    return dict(cap=rng.choice((0.0, 0.0, 20.0, 50.0)), slopes=rng.random() < 0.3,
                window=rng.choice((0, 0, 0, _log_uniform(rng, 1, most + 1))),
                prefix=rng.choice((0, 0, 0, _log_uniform(rng, 1, most))))


def _lengths(case):
    """(tokens held before, new tokens) of each request, by the case alone."""
    rng, R = random.Random(case["mix"]), case["R"]
    got = []
    for r in range(R):
        if case["kind"] == "append":
            n = case["new"] if R == 1 else max(1, case["new"] - rng.randrange(0, case["new"] // 2 + 1))
            got.append((case["most"] - n if R == 1 else _log_uniform(rng, 1, case["most"]), n))
        elif case["kind"] == "pages":
            n = case["new"] if R == 1 else _log_uniform(rng, 1, case["new"])
            got.append((case["most"] - n if R == 1 else _log_uniform(rng, 1, case["most"]), max(1, n)))
        else:
            n = 1 if r < case["single"] else case["new"]
            total = case["most"] if R == 1 else max(n, _log_uniform(rng, case["least"], case["most"]))
            got.append((max(n, total) - n, n))
    return got


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generator(seed, *ids):
    g = torch.Generator(device="cuda")
    s = seed % (1 << 40)
    for i in ids:
        s = s * 1009 + i + 1
    g.manual_seed(s % (1 << 62))
    return g


def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _large(D):
    """Keys have some features that are larger than the others."""
    f = torch.ones(D, device="cuda")
    f[::29] = 10.0
    return f


def _scale_for(top, fmt):
    """The least power of two whose multiple by the largest code reaches `top` (2^-100 at least)."""
    m, e = torch.frexp(top)
    whole, bits = (1.984375, 6) if fmt == "int8" else (1.75, 8)
    e = e - 1 - bits + (2.0 * m > whole)
    return torch.ldexp(torch.ones_like(top), torch.clamp(torch.where(top > 0, e, -100), min=-100))


def _held(g, fmt, dt, pages, kv, P, D):
    """A cache's content: values in the activation type, held as codes with a scale a page and head."""
    st = {}
    for name, shape in (("k", (pages, kv, P, D)), ("v", (pages, kv, D, P))):
        x = _randn(g, *shape).to(dt).float()
        if name == "k":
            x = x * _large(D)
        scale = _scale_for(x.abs().amax(dim=(2, 3)), fmt)
        c = x / scale[:, :, None, None]
        st["c" + name] = (torch.round(c) if fmt == "int8" else c).to(_HELD[fmt])
        st[name + "_scale"] = scale
    return st


def _frequencies(case):
    """Turns a position, in 64 bits: base^(-2i/rot), those of few turns in the first context slower."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64)
    f = _BASE ** (-2.0 * i / case["rot"]) / (2.0 * math.pi)
    share = torch.clamp((f * _CONTEXT - _LOW) / (_HIGH - _LOW), 0.0, 1.0)
    return f * (share + (1.0 - share) / case["factor"])


def _magnitude(case):
    return 1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0


def _inputs(case, seed):
    """Everything that a pass reads, by the seed alone (the lengths by the case)."""
    g, lengths, P, R = _generator(seed, 3), _lengths(case), case["P"], case["R"]
    kind, T = case["kind"], sum(n for _, n in lengths) + case.get("pad", 0)
    st = dict(T=T, held=_ints([h for h, _ in lengths]), fresh=_ints([n for _, n in lengths]))
    had, has = [-(-h // P) for h, _ in lengths], [-(-(h + n) // P) for h, n in lengths]
    wide = max(has)
    if kind in ("pages", "step"):
        pool = sum(has) + 5
        perm = torch.randperm(pool, device="cuda", generator=g).to(torch.int32)
        table = torch.full((R, wide + 1), -1, dtype=torch.int32)
        order, at = perm.cpu(), 0
        for r in range(R):
            table[r, :had[r]] = order[at:at + had[r]]
            at += had[r]
        free = perm[at:at + max(1, sum(has) - at - case["short"])] if case.get("short") else perm[at:]
        st.update(pool=pool, table=table.cuda(), free=free.contiguous())
    if kind == "pages":
        return st
    dt, D, kv, H = _DT[case["dtype"]], case["D"], case["kv"], case["heads"]
    st["q"] = _randn(g, T, H, D).to(dt)
    if kind in ("append", "step"):
        st["k"] = (_randn(g, T, kv, D) * _large(D)).to(dt)
        st["v"] = (_randn(g, T, kv, D) * (0.5 + 2.0 * torch.rand(T, 1, 1, device="cuda", generator=g))).to(dt)
    if kind == "append":
        # the pages that the new tokens touch, in random order, and every token in them
        touched = [-(-(h + n) // P) - h // P for h, n in lengths]
        st["pool"] = sum(touched) + 3
        order, at, slots, pos, live = torch.randperm(st["pool"], device="cuda", generator=g).tolist(), 0, [], [], []
        for (h, n), t in zip(lengths, touched):
            place = lambda p: order[at + p // P - h // P] * P + p % P  # noqa: E731
            slots += [place(p) for p in range(h, h + n)]
            live += [place(p) for p in range(h // P * P, h + n)]
            pos += range(h, h + n)
            at += t
        st.update(slots=_ints(slots), positions=_ints(pos), live=_ints(live))
    if kind == "attend":
        st["pool"] = sum(has) + 2
        order, at = torch.randperm(st["pool"], device="cuda", generator=g).to(torch.int32).cpu(), 0
        table = torch.zeros((R, wide), dtype=torch.int32)
        for r in range(R):
            table[r, :has[r]] = order[at:at + has[r]]
            at += has[r]
        starts = [0]
        for _, n in lengths:
            starts.append(starts[-1] + n)
        st.update(table=table.cuda(), starts=_ints(starts), lens=_ints([h + n for h, n in lengths]))
        if case["slopes"]:
            st["slopes"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H)
        if case["prefix"]:
            first = torch.randint(0, case["prefix"] + 1, (R,), device="cuda", generator=g)
            st["prefix"] = torch.minimum(first.to(torch.int32), st["lens"])
    st.update(_held(g, case["fmt"], dt, st["pool"], kv, P, D))
    return st


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    if own:
        _keep(st)
    elif case["kind"] in ("append", "step"):
        st["turns"] = _frequencies(case).cuda()
    return st


def _keep(st):
    """What a program keeps beside its tensors: the cache's and the batch's descriptions, the rotary
    frequencies, output buffers and workspace, and the plan that all layers of a step share (made here
    where the pass is one layer's call, in the pass where it is a step)."""
    from paper_2606_11244_amd import kv
    case, T = st["case"], st["T"]
    kind, st["kv"] = case["kind"], kv
    most = max(n for _, n in _lengths(case))

    def ints(n):
        return torch.empty(n, dtype=torch.int32, device="cuda")

    if kind in ("pages", "step"):
        st["batch"] = kv.Batch(st["table"], T, max_new=most)
        st["slots"], st["positions"], st["taken"] = ints(T), ints(T), ints(2)
    if kind == "pages":
        return
    dt, D = _DT[case["dtype"]], case["D"]
    st["cache"] = kv.Cache(st["ck"], st["cv"], st["k_scale"], st["v_scale"], dt)
    if kind in ("append", "step"):
        st["rope"] = kv.Rope(case["rot"], base=_BASE, interleaved=case["inter"], factor=case["factor"],
                             context=_CONTEXT, low_turns=_LOW, high_turns=_HIGH, magnitude=_magnitude(case))
        st["q_out"] = torch.empty_like(st["q"])
        n = st["live"].numel() if kind == "append" else T
        st["k_out"], st["v_out"] = (torch.empty((n, case["kv"], D), dtype=dt, device="cuda") for _ in range(2))
    if kind in ("attend", "step"):
        if kind == "attend":
            st["batch"] = kv.Batch(st["table"], T, max_new=most, starts=st["starts"], lens=st["lens"])
        st["plan"] = kv.AttentionPlan(st["cache"], st["batch"], case["heads"], window=case["window"],
                                      prefix=st.get("prefix"))
        st["out"] = torch.empty_like(st["q"])
        st["ws"] = torch.zeros(kv.attention_workspace(st["plan"]), dtype=torch.uint8, device="cuda")
    if kind == "attend":
        kv.attention_plan(st["plan"])


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _formulas(state)


def _run_own(st):
    kv, kind = st["kv"], st["case"]["kind"]
    if kind == "pages":
        return _own_pages(kv, st)
    if kind == "append":
        return _own_append(kv, st, st["live"])
    if kind == "attend":
        return _own_attention(kv, st, st["q"])
    out = _own_pages(kv, st)
    kv.attention_plan(st["plan"])
    out += _own_append(kv, st, st["slots"])
    return out + _own_attention(kv, st, st["q_out"])


def _own_pages(kv, st):
    b = st["batch"]
    kv.pages(b, st["held"], st["fresh"], st["free"], st["slots"], st["positions"], st["taken"],
             page_tokens=st["case"]["P"])
    return [b.starts, b.lens, b.table, st["slots"], st["positions"], st["taken"]]


def _own_append(kv, st, live):
    kv.append(st["cache"], st["k"], st["v"], st["slots"], st["positions"], rope=st["rope"], q=st["q"],
              q_out=st["q_out"])
    kv.read(st["cache"], live, st["k_out"], st["v_out"])
    return [st["q_out"], st["k_out"], st["v_out"], st["k_scale"], st["v_scale"]]


def _own_attention(kv, st, q):
    kv.attention(st["plan"], q, st["out"], softcap=st["case"]["cap"], slopes=st.get("slopes"),
                 workspace=st["ws"])
    return [st["out"]]


def _formulas(st):
    kind = st["case"]["kind"]
    if kind == "pages":
        return _plain_pages(st)
    if kind == "append":
        return _plain_append(st, st["slots"], st["positions"], st["live"])
    if kind == "attend":
        return _plain_attention(st, st["q"], st["starts"], st["lens"], st["table"])
    out = _plain_pages(st)
    starts, lens, table, slots, positions, _ = out
    out = out + _plain_append(st, slots, positions, slots)
    return out + _plain_attention(st, out[6], starts, lens, table)


def _plain_pages(st):
    P, T = st["case"]["P"], st["T"]
    h, n, table, free = st["held"].long(), st["fresh"].long(), st["table"].long(), st["free"].long()
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    starts = torch.cat((zero, torch.cumsum(n, 0)))
    had, has = (h + P - 1) // P, (h + n + P - 1) // P
    fill = torch.cumsum(has - had, 0)
    served = (fill <= free.numel()) | (has == had)
    taken = torch.where(served & (has > had), fill, torch.zeros_like(fill)).max()
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    take = (col >= had[:, None]) & (col < has[:, None]) & served[:, None]
    nth = (fill - (has - had) - had)[:, None] + col
    table = torch.where(take, free[torch.clamp(nth, 0, free.numel() - 1)], table)
    t = torch.arange(T, device="cuda")
    r = torch.clamp((t[:, None] >= starts[None, 1:]).sum(dim=1), max=h.numel() - 1)
    pos = h[r] + t - starts[r]
    live = (t < starts[-1]) & served[r]
    pos = torch.where(live, pos, torch.zeros_like(pos))
    slots = torch.where(live, table[r, pos // P] * P + pos % P, torch.full_like(pos, -1))
    lens = torch.where(served, h + n, torch.zeros_like(h))
    count = torch.stack((taken, (~served).sum()))
    return [v.to(torch.int32) for v in (starts, lens, table, slots, pos, count)]


def _plain_rope(st, x, positions):
    """In 64 bits: angles of far positions, and keys next to a border of two codes."""
    case, rot, x = st["case"], st["case"]["rot"], x.double()
    turn = positions.double()[:, None] * st["turns"][None, :]
    angle = ((turn - torch.floor(turn)) * (2.0 * math.pi))[:, None, :]
    c, s = (_magnitude(case) * f(angle) for f in (torch.cos, torch.sin))
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["inter"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack((a, b), dim=-1).flatten(2) if case["inter"] else torch.cat((a, b), dim=-1)
    return torch.cat((turned, x[..., rot:]), dim=-1)


def _plain_codes(c, fmt):
    return (torch.round(c) if fmt == "int8" else c.float()).to(_HELD[fmt])


def _plain_write(st, name, x, slots, token_dim):
    """New rows x [T][kv][D] into the pages of st["c" + name], scales and older codes as they have to be."""
    case, codes, scale = st["case"], st["c" + name], st[name + "_scale"]
    fmt, P, kv = case["fmt"], case["P"], case["kv"]
    page, at = slots.long() // P, slots.long() % P
    first = torch.full((codes.shape[0],), P, device="cuda").scatter_reduce(0, page, at, "amin")
    top = torch.zeros(scale.shape, dtype=x.dtype, device="cuda")
    top = top.scatter_reduce(0, page[:, None].expand(-1, kv), x.abs().amax(dim=2), "amax")
    need = _scale_for(top, fmt).float()
    keep = (first > 0)[:, None]
    new = torch.where((first < P)[:, None], torch.where(keep, torch.maximum(scale, need), need), scale)
    ratio = torch.where(keep, scale / new, torch.ones_like(new))[:, :, None, None]
    token = torch.arange(P, device="cuda").view((1, 1, P, 1) if token_dim == 2 else (1, 1, 1, P))
    old = codes.float()
    older = torch.where(token < first[:, None, None, None], old * ratio, old)
    codes.copy_(_plain_codes(older, fmt))
    scale.copy_(new)
    s = new[page][:, :, None].to(x.dtype)
    reach = torch.finfo(_DT[case["dtype"]]).max
    most = torch.where(s * _TOP[fmt] > reach, 63.0 if fmt == "int8" else 240.0, _TOP[fmt])
    c = _plain_codes(torch.minimum(torch.maximum(x / s, -most), most), fmt).view(torch.uint8)
    raw = codes.view(torch.uint8)
    if token_dim == 2:
        raw[page, :, at] = c
    else:
        raw[page, :, :, at] = c


def _plain_append(st, slots, positions, live):
    dt = _DT[st["case"]["dtype"]]
    _plain_write(st, "k", _plain_rope(st, st["k"], positions), slots, 2)
    _plain_write(st, "v", st["v"].float(), slots, 3)
    page, at = live.long() // st["case"]["P"], live.long() % st["case"]["P"]
    k = st["ck"].view(torch.uint8)[page, :, at].view(st["ck"].dtype).float() * st["k_scale"][page][:, :, None]
    v = st["cv"].view(torch.uint8)[page, :, :, at].view(st["cv"].dtype).float() * st["v_scale"][page][:, :, None]
    return [_plain_rope(st, st["q"], positions).to(dt), k.to(dt), v.to(dt), st["k_scale"], st["v_scale"]]


def _plain_gather(st, table):
    """K and V of every request, padded to the longest: [R][kv][L][D] in 32 bits."""
    case = st["case"]
    R, kv, P, D = case["R"], case["kv"], case["P"], case["D"]
    page = torch.clamp(table.long()[:, :-(-max(h + n for h, n in _lengths(case)) // P)], min=0)
    k = st["ck"].view(torch.uint8)[page].view(st["ck"].dtype).float() * st["k_scale"][page][..., None, None]
    v = st["cv"].view(torch.uint8)[page].view(st["cv"].dtype).float() * st["v_scale"][page][..., None, None]
    return k.transpose(1, 2).reshape(R, kv, -1, D), v.permute(0, 2, 1, 4, 3).reshape(R, kv, -1, D)


def _plain_attention(st, q, starts, lens, table):
    case = st["case"]
    R, kv, H, D = case["R"], case["kv"], case["heads"], case["D"]
    most, g = max(n for _, n in _lengths(case)), case["heads"] // case["kv"]
    k, v = _plain_gather(st, table)
    n = (starts[1:] - starts[:-1]).long()
    row = torch.arange(most, device="cuda")[None, :]
    token = torch.clamp(starts[:-1, None].long() + row, max=q.shape[0] - 1)
    i = (lens.long() - n)[:, None] + row                                   # position of each row
    qs = q.float()[token].view(R, most, kv, g, D).permute(0, 2, 3, 1, 4)     # [R][kv][g][most][D]
    s = torch.matmul(qs.reshape(R, kv, g * most, D), k.transpose(2, 3).contiguous()).view(R, kv, g, most, -1)
    s = s / math.sqrt(D)
    if case["cap"]:
        s = case["cap"] * (1.0 - 2.0 / (torch.exp(2.0 * s / case["cap"]) + 1.0))
    j = torch.arange(s.shape[-1], device="cuda")[None, None, :]
    far = i[:, :, None] - j
    if case["slopes"]:
        s = s - st["slopes"].view(1, kv, g, 1, 1) * far.abs().float()[:, None, None]
    seen = far >= 0
    if case["window"]:
        seen = seen & (far < case["window"])
    if case["prefix"]:
        seen = seen | (j < st["prefix"][:, None, None])
    seen = (seen & (j < lens[:, None, None]))[:, None, None]
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.reshape(R, kv, g * most, -1), v).view(R, kv, g, most, D)
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    o = o.permute(0, 3, 1, 2, 4).reshape(R, most, H, D)
    t = torch.arange(q.shape[0], device="cuda")
    r = (t[:, None] >= starts[None, 1:]).sum(dim=1)
    return [o[r, t - starts.long()[r]].to(q.dtype)]


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def _seen(case, h, n):
    """Keys that any row of a request sees, and pairs of a row and a key it sees (a prefix: half of
    what it may be, as it is drawn)."""
    w, half = case["window"] or h + n, min(case["prefix"] // 2, h + n)
    first = max(0, h - w + 1)
    pairs = sum(min(i + 1, w) + min(half, max(0, i + 1 - w)) for i in range(h, h + n))
    return h + n - first + min(first, half), pairs


def work(case):
    P, lengths, kind = case["P"], _lengths(case), case["kind"]
    T, R, b, f = sum(n for _, n in lengths), case["R"], 0, 0
    new_pages = sum(-(-(h + n) // P) - -(-h // P) for h, n in lengths)
    if kind in ("pages", "step"):
        b += 4 * (2 * R + 2 * R + 1 + 2 * (T + case.get("pad", 0)) + 2 * new_pages + 2)
    if kind == "pages":
        return {"bytes": b, "flops": 0}
    kv, D, H = case["kv"], case["D"], case["heads"]
    if kind in ("append", "step"):
        live = sum(h + n - h // P * P for h, n in lengths) if kind == "append" else T
        touched = sum(-(-(h + n) // P) - h // P for h, n in lengths)
        # queries both ways, keys and values, their codes; scales; the codes read back, their values
        b += T * D * (4 * H + 4 * kv + 2 * kv) + 16 * touched * kv + live * kv * D * 6 + 8 * T
        f += T * (3 * (H + kv) * case["rot"] + 4 * kv * D)
    if kind in ("attend", "step"):
        for h, n in lengths:
            keys, pairs = _seen(case, h, n)
            b += 2 * keys * kv * D + -(-keys // P) * (8 * kv + 4) + 4 * n * H * D
            f += 4 * pairs * H * D
    return {"bytes": b, "flops": f}


# ---------------------------------------------------------------------------
# the operators' definition in 64 bits: page by page, request by request
# ---------------------------------------------------------------------------

def _exact_codes(c, fmt):
    if fmt == "int8":
        return torch.round(c)
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(c.abs() + 1e-300)), min=-6.0) - 3.0)
    return torch.round(c / step) * step


def _exact_rope(case, x, positions):
    i = torch.arange(case["rot"], device="cuda")
    pair = i // 2 if case["inter"] else i % (case["rot"] // 2)
    other = i + 1 - 2 * (i % 2) if case["inter"] else (i + case["rot"] // 2) % case["rot"]
    sign = torch.where(other > i, -1.0, 1.0).double()
    turns = positions.double()[:, None] * _frequencies(case).cuda()[pair]
    angle = 2.0 * math.pi * torch.remainder(turns, 1.0)[:, None, :]
    y = x.double().clone()
    r = y[..., :case["rot"]]
    y[..., :case["rot"]] = _magnitude(case) * (r * torch.cos(angle) + sign * r[..., other] * torch.sin(angle))
    return y


def _exact_append(st, case, slots, positions):
    """Values and scales of K and V after the call, K and V as [pages][kv][P][D], and the turned queries."""
    P, fmt, got = case["P"], case["fmt"], []
    page, at = (slots // P).tolist(), (slots % P).tolist()
    rows = {}
    for t, p in enumerate(page):
        rows.setdefault(p, []).append(t)
    for name, x in (("k", _exact_rope(case, st["k"], positions)), ("v", st["v"].double())):
        codes = st["c" + name].float().double()
        codes = codes if name == "k" else codes.transpose(2, 3).contiguous()
        scale = st[name + "_scale"].double().clone()
        for p, ts in rows.items():
            new = x[ts].transpose(0, 1)                       # [kv][n][D]
            top = new.abs().amax(dim=(1, 2))
            s = torch.exp2(torch.ceil(torch.log2(torch.clamp(top / _TOP[fmt], min=2.0 ** -100))))
            first = at[ts[0]]
            if first:
                s = torch.maximum(s, scale[p])
                codes[p, :, :first] = _exact_codes(codes[p, :, :first] * (scale[p] / s)[:, None, None], fmt)
            codes[p, :, first:first + len(ts)] = _exact_codes(new / s[:, None, None], fmt)
            scale[p] = s
        got.append((codes * scale[:, :, None, None], scale))
    return got, _exact_rope(case, st["q"], positions)


def _exact_attention(st, case, q, k, v, lengths, table):
    P, kv, D, outs, t = case["P"], case["kv"], case["D"], [], 0
    g = case["heads"] // kv
    for r, (h, n) in enumerate(lengths):
        pages, L = table[r, :-(-(h + n) // P)].long(), h + n
        i, j = torch.arange(h, L, device="cuda")[:, None], torch.arange(L, device="cuda")[None, :]
        hidden = j > i
        if case["window"]:
            hidden = hidden | (i - j >= case["window"])
        if case["prefix"]:
            hidden = hidden & (j >= st["prefix"][r])
        heads = []
        for c in range(kv):
            kk = k[pages, c].reshape(-1, D)[:L].double()
            vv = v[pages, c].reshape(-1, D)[:L].double()
            for e in range(c * g, c * g + g):
                s = (q[t:t + n, e].double() @ kk.T) * D ** -0.5
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                if case["slopes"]:
                    s = s - st["slopes"][e].double() * (i - j).abs()
                heads.append(torch.softmax(s.masked_fill(hidden, -math.inf), dim=-1) @ vv)
        outs.append(torch.stack(heads, dim=1))
        t += n
    return torch.cat(outs)


def exact(case, seed):
    kind, lengths, P = case["kind"], _lengths(case), case["P"]
    if kind == "pages":
        return None
    st = _inputs(case, seed)
    if kind == "attend":
        k = st["ck"].float() * st["k_scale"][:, :, None, None]
        v = (st["cv"].float() * st["v_scale"][:, :, None, None]).transpose(2, 3)
        return [_exact_attention(st, case, st["q"], k, v, lengths, st["table"])]
    if kind == "append":
        slots, live, positions = st["slots"], st["live"], st["positions"]
    else:
        table, free = st["table"].clone(), st["free"].tolist()
        for r, (h, n) in enumerate(lengths):
            for p in range(-(-h // P), -(-(h + n) // P)):
                table[r, p] = free.pop(0)
        positions = _ints([p for h, n in lengths for p in range(h, h + n)])
        slots = live = _ints([int(table[r, p // P]) * P + p % P for r, (h, n) in enumerate(lengths) for p in range(h, h + n)])
    ((k, ks), (v, vs)), q = _exact_append(st, case, slots, positions)
    page, at = live.long() // P, live.long() % P
    out = [q, k[page, :, at], v[page, :, at], ks, vs]
    if kind == "append":
        return out
    # attention reads the queries as they are held, rounded to the activation type
    return [None] * 6 + out + [_exact_attention(st, case, q.to(_DT[case["dtype"]]), k, v, lengths, table)]
