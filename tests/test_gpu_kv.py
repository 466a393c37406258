"""Attention over a paged cache held in 8 bits, on the GPU, against plain
references in 64 bits: block tables and slots, rotary positions with the
cache's writing, values back, attention, and a run of them together."""
from __future__ import annotations

import random

import pytest
import torch

import kv_util as U

pytestmark = pytest.mark.gpu

ACTS = [torch.float16, torch.bfloat16]
CODES = [torch.int8, torch.float8_e4m3fn]
FAR = 2 ** 31 - 1


def _kv():
    from paper_2606_11244_amd import kv
    return kv


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------
# block tables, slots, positions
# ---------------------------------------------------------------------------

def _run_pages(held, fresh, free, table, tokens, P, ld=None):
    kv = _kv()
    R, width = len(held), len(table[0]) if table else 4
    full = torch.full((max(R, 1), ld or width), -7, dtype=torch.int32, device="cuda")
    t = full[:R, :width]
    if R:
        t.copy_(_ints(table))
    b = kv.Batch(t, tokens, max_new=max(1, tokens))
    b.starts.fill_(-9)
    slots, pos, taken = (torch.full((n,), -9, dtype=torch.int32, device="cuda") for n in (tokens, tokens, 2))
    kv.pages(b, _ints(held), _ints(fresh), _ints(free), slots, pos, taken, page_tokens=P)
    got = [x.tolist() for x in (b.starts, b.lens, t, slots, pos, taken)]
    assert bool((full[:, width:] == -7).all())
    want = U.plain_pages(held, fresh, free, table, tokens, P)
    for name, g, w in zip(("starts", "lens", "table", "slots", "positions", "taken"), got, want):
        assert g == list(w), name
    return got


@pytest.mark.parametrize("R,P,most,new,short,pad", [
    (1, 16, 1, 1, 0, 0), (1, 64, 700, 300, 0, 3), (5, 32, 100, 40, 0, 0), (5, 16, 100, 40, 4, 9),
    (64, 128, 3000, 1, 0, 0), (200, 16, 500, 30, 60, 64), (1025, 32, 200, 3, 0, 1), (4096, 64, 130, 2, 500, 0)])
def test_pages(R, P, most, new, short, pad):
    rng = random.Random(R * 31 + P)
    held = [rng.randrange(0, most + 1) for _ in range(R)]
    fresh = [rng.choice((0, 1, new, rng.randrange(0, new + 1))) for _ in range(R)]
    width = -(-(most + new) // P) + 1
    ids = list(range(R * width + 8))
    rng.shuffle(ids)
    table = [[ids.pop() if j < -(-h // P) else -1 for j in range(width)] for h in held]
    need = sum(-(-(h + f) // P) - -(-h // P) for h, f in zip(held, fresh))
    _run_pages(held, fresh, ids[:max(0, need - short)], table, sum(fresh) + pad, P, ld=width + 3)


def test_pages_that_cannot_be_served():
    P, width = 16, 4
    table = [[10 * r + j for j in range(width)] for r in range(7)]
    #        ok, negative, too long, row of the table too short, ok, no pages left, needs none
    held = [3, -1, 2 ** 30, 60, 0, 16, 5]
    fresh = [2, 4, 1, 5, 33, 40, 2]
    got = _run_pages(held, fresh, [90, 91, 92], table, 100, P)
    assert got[1] == [5, 0, 0, 0, 33, 0, 7] and got[5] == [3, 4]
    # rows past the step's tokens, and what comes after them
    _run_pages([0, 0, 0], [10, 20, 1], list(range(5)), [[-1] * 4] * 3, 29, P)
    _run_pages([0, 0], [2 ** 30, 1], list(range(5)), [[-1] * 4] * 2, 29, P)
    _run_pages([0] * 3, [2 ** 31 - 1] * 3, [1], [[-1] * 4] * 3, 5, P)
    # negative table entries and slots past 31 bits have no slot
    _run_pages([3, 3], [1, 1], [], [[-5] * 4, [2 ** 28] * 4], 2, P)
    _run_pages([], [], [], [], 7, P)
    _run_pages([4], [0], [1], [[3] * 4], 0, P)


# ---------------------------------------------------------------------------
# rotary positions and the cache's writing
# ---------------------------------------------------------------------------

def _content(cache):
    """((K codes, scales), (V codes as [pages][kv][P][D], scales)) in 64 bits, on the CPU."""
    return ((U.codes_of(cache.k), cache.k_scale.cpu().double()),
            (U.codes_of(cache.v).transpose(2, 3).contiguous(), cache.v_scale.cpu().double()))


def _random_cache(kv, pages, heads, P, D, act, codes, seed):
    """A cache of arbitrary codes (no NaN) and scales."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = kv.new_cache(pages, heads, P, D, act, codes)
    for t in (c.k, c.v):
        t.view(torch.int8).copy_(torch.randint(-127, 127, t.shape, device="cuda", generator=g, dtype=torch.int8))
        if codes is torch.float8_e4m3fn:
            t.view(torch.uint8)[t.view(torch.uint8) & 0x7F == 0x7F] = 0
    for s in (c.k_scale, c.v_scale):
        s.copy_(torch.exp2(torch.randint(-9, -3, s.shape, device="cuda", generator=g).float()))
    return c


def _append_checked(cache, rope, interleaved, magnitude, q, k, v, slots, positions, in_place=False):
    kv = _kv()
    rot = rope.c.rotary_dim if rope else 0
    freqs = [f % 2 ** 64 for f in rope.freqs.tolist()] if rope else []
    before = _content(cache)
    q_out = None if q is None else (q if in_place else torch.full_like(q, 7.0))
    q0 = None if q is None else q.clone()
    kv.append(cache, k, v, _ints(slots), _ints(positions), rope=rope, q=q, q_out=q_out)
    after = _content(cache)
    P, act, codes = cache.page_tokens, cache.act_dtype, cache.k.dtype
    x = U.turned(k.cpu(), positions, freqs, rot, interleaved, magnitude)
    # an angle is off by 2^-32 of a turn and its rounding, cosine and sine by 2^-24 and 3e-8, four products
    # and sums: 2^-21 of the pair's length in all
    length = k.cpu().double().abs().amax(dim=2, keepdim=True) * 2 * abs(magnitude) * 2.0 ** -21
    slack = length.expand_as(x).clone()
    slack[:, :, rot:] = 0
    U.check_written(before[0], after[0], x, slots, P, codes, act, slack)
    U.check_written(before[1], after[1], v.cpu().double(), slots, P, codes, act, torch.zeros_like(x))
    if q is not None:
        want = U.turned(q0.cpu(), positions, freqs, rot, interleaved, magnitude)
        length = q0.cpu().double().abs().amax(dim=2, keepdim=True) * 2 * abs(magnitude) * 2.0 ** -21
        live = torch.tensor([0 <= s < cache.k.shape[0] * P for s in slots])
        d = (q_out.cpu().double() - want).abs()
        assert bool((d <= U.U[act] * want.abs() + length + 2.0 ** -25)[live].all()), d[live].max()
        rest = q0.cpu() if in_place else torch.full_like(q0, 7.0).cpu()
        assert torch.equal(q_out.cpu()[~live], rest[~live])
        assert torch.equal(q_out.cpu()[live][:, :, rot:], q0.cpu()[live][:, :, rot:])


def _rope(kv, rot, interleaved, magnitude=1.0, factor=1.0):
    return kv.Rope(rot, 10000.0, interleaved=interleaved, magnitude=magnitude, factor=factor, context=4096)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("codes", CODES)
@pytest.mark.parametrize("P,D,heads,kvh,rot,interleaved", [
    (16, 64, 4, 2, 64, False), (16, 128, 3, 1, 128, True), (32, 128, 10, 5, 32, True), (64, 64, 7, 7, 16, False),
    (128, 128, 8, 8, 128, False), (32, 64, 6, 3, 6, True), (64, 128, 2, 2, 50, False), (16, 64, 1, 1, 0, False)])
def test_append(act, codes, P, D, heads, kvh, rot, interleaved):
    kv = _kv()
    g = torch.Generator(device="cuda").manual_seed(P + D + rot)
    cache = _random_cache(kv, 40, kvh, P, D, act, codes, 3)
    rope = _rope(kv, rot, interleaved, 1.25, 8.0) if rot else None

    def new(n, size=1.0):
        # rows of a packed projection: q, k and v beside each other
        x = (torch.randn(n, heads + 2 * kvh, D, device="cuda", generator=g) * size).to(act)
        return x[:, :heads], x[:, heads:heads + kvh], x[:, heads + kvh:]

    # a prompt over several pages, from the middle of one; another one; padding between them
    n1, n2, at = P + P // 2 + 5, 3, 5
    place = lambda p: (11 + 3 * (p // P)) * P + p % P  # noqa: E731
    slots = [place(at + i) for i in range(n1)] + [-1, 40 * P, FAR] + [2 * P + i for i in range(n2)]
    pos = [at + i for i in range(n1)] + [0, 5, FAR] + [1000000 + i for i in range(n2)]
    _append_checked(cache, rope, interleaved, 1.25 if rot else 1.0, *new(n1 + 3 + n2), slots, pos)
    # one token each, larger and smaller ones by turns: scales that grow, and stay
    for step, size in enumerate((0.01, 3.0, 1.0, 40.0, 7.0, 300.0)):
        slots = [place(at + n1 + step), 2 * P + n2 + step, 7 * P + step]
        pos = [at + n1 + step, 1000000 + n2 + step, 2 ** 30 - 7 + step]
        _append_checked(cache, rope, interleaved, 1.25 if rot else 1.0, *new(3, size), slots, pos, in_place=step == 3)
    q, k, v = new(2)
    _append_checked(cache, rope, interleaved, 1.25 if rot else 1.0, None, k, v, [P - 1, 39 * P], [4, 0])


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("codes", CODES)
def test_append_of_many_tokens(act, codes):
    """More rows than a workgroup's window: the runs of several windows and of single tokens."""
    kv = _kv()
    g = torch.Generator(device="cuda").manual_seed(9)
    P, D = 32, 64
    cache = _random_cache(kv, 80, 2, P, D, act, codes, 5)
    order = list(range(80))
    random.Random(4).shuffle(order)
    slots, pos = [], []
    for r in range(12):  # prompts of 90 tokens from place 7r of their first page, three pages or four each
        ids = order[6 * r:6 * r + 6]
        slots += [ids[p // P] * P + p % P for p in range(7 * r % P, 7 * r % P + 90)]
        pos += list(range(7 * r % P, 7 * r % P + 90))
    slots += [ids * P + ids % P for ids in order[72:]]
    pos += [100 + i for i in range(8)]
    T = len(slots)
    k, v, q = (torch.randn(T, h, D, device="cuda", generator=g).to(act) for h in (2, 2, 4))
    assert T > 1024
    _append_checked(cache, _rope(kv, 64, False), False, 1.0, q, k, v, slots, pos)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("codes", CODES)
@pytest.mark.parametrize("rot,interleaved", [(64, False), (32, True), (50, True)])
def test_keys_have_the_nearest_codes(act, codes, rot, interleaved):
    """One rounding: a code is the nearest to the rotation in 64 bits, whose own error (that of an angle held
    as a 64-bit fraction, Taylor's sums and a dozen roundings, less than 2^-45 of a code) is all that is allowed."""
    kv = _kv()
    g = torch.Generator(device="cuda").manual_seed(rot)
    P, D, T = 64, 64, 4096
    cache = kv.new_cache(T // P, 2, P, D, act, codes)
    rope = _rope(kv, rot, interleaved)
    k = torch.randn(T, 2, D, device="cuda", generator=g).to(act)
    pos = torch.randint(0, 2 ** 30, (T,), device="cuda", generator=g, dtype=torch.int32)
    kv.append(cache, k, k.clone(), _ints(range(T)), pos, rope=rope)
    x = U.turned(k.cpu(), pos.tolist(), [f % 2 ** 64 for f in rope.freqs.tolist()], rot, interleaved, 1.0)
    (have, scale), _ = _content(cache)
    have = have.transpose(1, 2).reshape(T, 2, D)
    c = x / scale.repeat_interleave(P, 0)[:, :, None]
    c = c.clamp(-U.TOP[codes], U.TOP[codes])
    step = U.step_of(c, codes)
    assert bool(((have - c).abs() <= 0.5 * step + 2.0 ** -45 * c.abs()).all())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("codes", CODES)
def test_append_at_the_ends_of_the_range(act, codes):
    kv = _kv()
    P, D, inf, nan = 16, 64, float("inf"), float("nan")
    top = float(torch.finfo(act).max)
    cache = kv.new_cache(8, 1, P, D, act, codes)
    for slot, values in ((0, [0.0]), (1, [0.0]), (P, [top, -top, 1.0]), (2 * P, [inf, -inf, nan, 3.0]),
                         (3 * P, [nan]), (4 * P, [1e-7]), (4 * P + 1, [top]), (5 * P, [127.0, -127.0]),
                         (6 * P, [448.0]), (7 * P, [1.0]), (7 * P + 1, [-448.0])):
        x = torch.zeros(1, 1, D, device="cuda")
        x[0, 0, 3:3 + len(values)] = torch.tensor(values, device="cuda")
        x = x.to(act)
        _append_checked(cache, None, False, 1.0, None, x, x.clone(), [slot], [0])
    ko, vo = (torch.empty(8 * P, 1, D, dtype=act, device="cuda") for _ in range(2))
    kv.read(cache, torch.arange(8 * P, dtype=torch.int32, device="cuda"), ko, vo)
    assert bool(torch.isfinite(ko.float()).all()) and torch.equal(ko, vo)
    assert ko[2 * P, 0, 3:7].tolist() == [U.TOP[codes] * float(cache.k_scale[2, 0]), -U.TOP[codes] * float(cache.k_scale[2, 0]), 0.0, 3.0]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("codes", CODES)
@pytest.mark.parametrize("P,D,kvh,n", [(16, 64, 1, 1), (64, 128, 3, 77), (128, 64, 8, 16)])
def test_read(act, codes, P, D, kvh, n):
    kv = _kv()
    cache = _random_cache(kv, 9, kvh, P, D, act, codes, n)
    rng = random.Random(n)
    slots = [rng.randrange(0, 9 * P) for _ in range(n)]
    slots[n // 2] = rng.choice((-1, 9 * P, FAR)) if n > 1 else slots[0]
    ko, vo = (torch.full((n, kvh, D), 5.0, dtype=act, device="cuda") for _ in range(2))
    kv.read(cache, _ints(slots), ko, vo)
    for (c, s), got in zip(_content(cache), (ko, vo)):
        for i, slot in enumerate(slots):
            want = torch.full((kvh, D), 5.0) if not 0 <= slot < 9 * P else c[slot // P, :, slot % P] * s[slot // P][:, None]
            assert torch.equal(got[i].cpu().double(), want.double()), i


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

class Setup:
    """Requests of lengths (rows, tokens in the cache) on a cache of random content."""

    def __init__(self, lengths, heads, kvh, D, P, act, codes, seed=1, pad=0, max_new=None, window=0, prefix=None,
                 poison=True):
        kv = self.kv = _kv()
        rng, g = random.Random(seed), torch.Generator(device="cuda").manual_seed(seed)
        self.lengths, self.heads = lengths, heads
        need = [-(-max(L, 1) // P) for _, L in lengths]
        self.pool = sum(need) + 3
        self.cache = _random_cache(kv, self.pool, kvh, P, D, act, codes, seed)
        ids = list(range(self.pool))
        rng.shuffle(ids)
        self.table = [[ids.pop() for _ in range(n)] for n in need]
        wide = max(need) + 1
        if poison:  # what no token's value is: bytes behind the last token, scales of pages without one
            used = {p for row, (_, L) in zip(self.table, lengths) for p in row[:-(-L // P)]}
            bad = torch.tensor([p not in used for p in range(self.pool)], device="cuda")
            for s in (self.cache.k_scale, self.cache.v_scale):
                s[bad] = float("nan")
            for row, (_, L) in zip(self.table, lengths):
                if L % P:
                    for t in (self.cache.k.view(torch.uint8)[row[L // P], :, L % P:], self.cache.v.view(torch.uint8)[row[L // P], :, :, L % P:]):
                        t.fill_(0x7F if codes is torch.float8_e4m3fn else 0x80)
        self.starts = [0]
        for n, _ in lengths:
            self.starts.append(self.starts[-1] + n)
        T = self.starts[-1] + pad
        self.q = torch.randn(T, heads, D, device="cuda", generator=g).to(act)
        self.out = torch.full_like(self.q, 9.0)
        table = _ints([row + [-1] * (wide - len(row)) for row in self.table])
        self.lens = [L for _, L in lengths]
        self.batch = kv.Batch(table, T, max_new=max_new or max(1, max(n for n, _ in lengths)), starts=_ints(self.starts),
                              lens=_ints(self.lens))
        self.window, self.prefix, self.max_new = window, prefix, max_new
        self.plan = kv.AttentionPlan(self.cache, self.batch, heads, window=window,
                                     prefix=None if prefix is None else _ints(prefix))
        self.ws = torch.zeros(kv.attention_workspace(self.plan), dtype=torch.uint8, device="cuda")

    def run(self, **kw):
        self.kv.attention_plan(self.plan)
        self.kv.attention(self.plan, self.q, self.out, workspace=self.ws, **kw)
        return self.out

    def gathered(self):
        got = []
        P = self.cache.page_tokens
        for c, s in _content(self.cache):
            x = c * torch.nan_to_num(s, nan=1.0)[:, :, None, None]
            got.append([x[row].transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :L].transpose(0, 1)
                        for row, L in zip(self.table, self.lens)])
        return got, P

    def check(self, scale=None, softcap=0.0, slopes=None, dead=None):
        self.run(scale=scale, softcap=softcap, slopes=slopes)
        (k, v), _ = self.gathered()
        scale = self.cache.head_dim ** -0.5 if scale is None else scale
        want, bound = U.plain_attention(self.q.cpu(), k, v, self.starts, self.lens, self.heads, scale=scale,
                                        softcap=softcap, slopes=None if slopes is None else slopes.tolist(),
                                        window=self.window, prefix=self.prefix, dead=dead, max_new=self.max_new)
        got = self.out.cpu().double()
        for r, (n, _) in enumerate(self.lengths):
            rows = slice(self.starts[r], self.starts[r] + min(n, self.max_new or n))
            d = (got[rows] - want[rows]).abs() - bound[rows]
            assert bool((d <= 0).all()), (r, self.lengths[r], float(d.max()), float(want[rows].abs().max()))
            untouched = got[self.starts[r] + min(n, self.max_new or n):self.starts[r + 1]]
            assert bool((untouched == 9.0).all())
        assert bool((got[self.starts[-1]:] == 9.0).all())


LENGTHS = {
    "one token": [(1, 1)],
    "a page's borders": [(1, L) for L in (15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129)],
    "decode": [(1, 700), (1, 3), (1, 2100), (1, 64), (1, 1)],
    "long": [(1, 9001), (1, 5)],
    "chunks": [(2, 2), (5, 300), (17, 17), (40, 41), (1, 90), (3, 1000)],
    "prompt": [(300, 300)],
    "prompt and decode": [(1, 500), (130, 700), (1, 1), (257, 257), (1, 130)],
}


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("codes", CODES)
@pytest.mark.parametrize("what", list(LENGTHS))
@pytest.mark.parametrize("heads,kvh,D,P", [(8, 2, 128, 64), (6, 6, 64, 16)])
def test_attention(act, codes, what, heads, kvh, D, P):
    Setup(LENGTHS[what], heads, kvh, D, P, act, codes, pad=2).check()


@pytest.mark.parametrize("heads,kvh", [(1, 1), (3, 1), (7, 1), (8, 1), (16, 1), (17, 1), (40, 1), (10, 5), (64, 8)])
@pytest.mark.parametrize("P", [16, 32, 128])
def test_attention_head_layouts(heads, kvh, P):
    Setup([(1, 200), (2, 150), (1, 31), (9, 77)], heads, kvh, 64, P, torch.bfloat16, torch.int8).check()
    Setup([(1, 333), (1, 1)], heads, kvh, 128, P, torch.float16, torch.float8_e4m3fn).check()


@pytest.mark.parametrize("act,codes", [(torch.float16, torch.float8_e4m3fn), (torch.bfloat16, torch.int8)])
@pytest.mark.parametrize("lengths", [[(1, 600), (1, 40), (1, 1)], [(200, 600), (1, 300), (33, 40)]])
@pytest.mark.parametrize("softcap,slopes,window,prefix", [
    (15.0, False, 0, False), (0.0, True, 0, False), (0.0, False, 1, False), (0.0, False, 100, False),
    (0.0, False, 10000, False), (0.0, False, 0, True), (5.0, True, 70, True)])
def test_attention_options(act, codes, lengths, softcap, slopes, window, prefix):
    heads, kvh = 6, 2
    s = torch.exp2(-torch.arange(1, heads + 1, device="cuda").float()) if slopes else None
    first = [min(37, L) for _, L in lengths] if prefix else None
    if prefix:
        first[-1] = lengths[-1][1]
    Setup(lengths, heads, kvh, 64, 32, act, codes, window=window, prefix=first).check(
        softcap=softcap, slopes=s, scale=0.3 if softcap else None)


def test_attention_prefixes_of_any_value():
    lengths = [(3, 100), (50, 80), (2, 20), (1, 9)]
    s = Setup(lengths, 4, 2, 64, 16, torch.float16, torch.int8, prefix=[-5, 2 ** 31 - 1, 0, 4], window=8)
    s.prefix = [0, 80, 0, 4]
    s.check()


def test_attention_of_requests_without_keys():
    """lens 0 (not served), fewer tokens than rows, no rows at all, table entries outside the pool."""
    s = Setup([(2, 40), (3, 0), (0, 50), (5, 2), (70, 0), (1, 200), (90, 20)], 4, 2, 64, 16, torch.float16,
              torch.float8_e4m3fn, pad=3)
    dead = [torch.zeros(max(L, 1), dtype=torch.bool) for _, L in s.lengths]
    for r, page, bad in ((0, 1, -1), (5, 0, s.pool), (5, 3, 2 ** 31 - 1), (5, 7, -2 ** 31)):
        s.batch.table[r, page] = bad
        dead[r][16 * page:16 * page + 16] = True
    s.check(dead=dead)
    assert bool((s.out[2:5] == 0).all()) and bool((s.out[5:8] == 0).all())
    # every page of a request outside the pool
    s.batch.table[5].fill_(s.pool + 5)
    dead[5][:] = True
    s.check(dead=dead)


def test_attention_of_more_rows_than_said():
    Setup([(5, 60), (1, 33), (3, 3)], 8, 2, 64, 16, torch.bfloat16, torch.int8, max_new=2).check()
    Setup([(300, 400), (1, 33)], 8, 2, 64, 16, torch.bfloat16, torch.int8, max_new=40).check()


def test_attention_of_starts_that_contradict_themselves():
    """Rows that no order makes sense of: nothing outside the step is touched, and what comes after is right."""
    act, codes = torch.bfloat16, torch.int8
    s = Setup([(3, 900), (40, 1200), (1, 2500), (2, 33)], 8, 1, 64, 16, act, codes, pad=4)
    want = s.run().clone()
    bad = [[46, 0, 46, 0, 46], [-5, 2 ** 31 - 1, 3, -2 ** 31, 50], [46, 46, 46, 46, 46], [0, 46, 46, 0, 46]]
    for starts in bad:
        s.batch.starts.copy_(_ints(starts))
        s.batch.lens.copy_(_ints([2 ** 31 - 1, 1200, -7, 2 ** 30]))
        s.run()
        s.batch.starts.copy_(_ints(s.starts))
        s.batch.lens.copy_(_ints(s.lens))
        s.out.fill_(9.0)
        assert torch.equal(s.run(), want)


def test_attention_strides():
    for lengths in ([(1, 300), (1, 20)], [(70, 300), (1, 20)]):
        s = Setup(lengths, 4, 2, 128, 32, torch.float16, torch.int8)
        want = s.run().clone()
        T, H, D = s.q.shape
        packed = torch.full((T, H + 4, D), 3.0, dtype=s.q.dtype, device="cuda")
        packed[:, :H] = s.q
        wide = torch.full((T, H + 1, D), 3.0, dtype=s.q.dtype, device="cuda")
        s.q, s.out = packed[:, :H], wide[:, :H]
        assert torch.equal(s.run(), want) and bool((wide[:, H:] == 3.0).all())


def test_attention_extreme_scores_and_values():
    """Scores of several thousands, values near the type's ends, a scale of zero, a page of zeros."""
    for act, codes in ((torch.float16, torch.int8), (torch.bfloat16, torch.float8_e4m3fn), (torch.float16, torch.float8_e4m3fn)):
        for lengths in ([(1, 500), (1, 70)], [(80, 500)]):
            s = Setup(lengths, 4, 1, 64, 16, act, codes)
            s.check(scale=8.0)
            s.check(scale=0.0)
            s.check(scale=-0.2)
            s.cache.v_scale[s.table[0][2]] = 2.0 ** -100
            s.cache.k_scale[s.table[0][3]] = 2.0 ** -100
            s.cache.v_scale[s.table[0][4]] = 2.0 ** 6
            s.cache.v.view(torch.uint8)[s.table[0][5]] = 0
            s.check()


@pytest.mark.parametrize("codes", CODES)
@pytest.mark.parametrize("act,size", [(torch.float16, 2.0 ** -24), (torch.float16, 2.0 ** -20), (torch.float16, 2.0 ** -14),
                                      (torch.bfloat16, 2.0 ** -90), (torch.float16, 3e4)])
@pytest.mark.parametrize("lengths", [[(1, 200)], [(20, 200)], [(400, 400)]])
def test_attention_of_values_at_the_ends_of_the_range(act, codes, size, lengths):
    """V of the type's least values (in fp16 of few steps of 2^-24) and of its largest, written and read."""
    s = Setup(lengths, 64 if lengths[0][0] == 400 else 4, 64 if lengths[0][0] == 400 else 1, 64, 16, act, codes)
    g = torch.Generator(device="cuda").manual_seed(3)
    L, kvh = lengths[0][1], s.cache.kv_heads
    slots = [s.table[0][j // 16] * 16 + j % 16 for j in range(L)]
    k = torch.randn(L, kvh, 64, device="cuda", generator=g).to(act)
    v = (torch.randn(L, kvh, 64, device="cuda", generator=g).clamp(-2, 2) * size).to(act)
    s.kv.append(s.cache, k, v, _ints(slots))
    s.check()
    assert bool(torch.isfinite(s.out.float()).all()) and (size < 2.0 ** -20 or bool((s.out != 0).any()))


# Steps of so many rows (padding counts: sizes alone are known to the host) that tiles are the large ones.
LARGE = dict(heads=64, pad=1600)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("codes", CODES)
@pytest.mark.parametrize("what", ["chunks", "prompt", "prompt and decode"])
@pytest.mark.parametrize("kvh,D,P", [(8, 128, 64), (4, 64, 16), (64, 128, 128), (1, 64, 32), (2, 128, 16)])
def test_attention_in_large_tiles(act, codes, what, kvh, D, P):
    Setup(LENGTHS[what], kvh=kvh, D=D, P=P, act=act, codes=codes, **LARGE).check()


@pytest.mark.parametrize("D,act,codes", [(128, torch.float16, torch.float8_e4m3fn), (64, torch.bfloat16, torch.int8),
                                         (128, torch.bfloat16, torch.float8_e4m3fn), (64, torch.float16, torch.int8)])
@pytest.mark.parametrize("softcap,slopes,window,prefix", [
    (15.0, False, 0, False), (0.0, True, 0, False), (0.0, False, 1, False), (0.0, False, 100, False),
    (0.0, False, 10000, False), (0.0, False, 0, True), (5.0, True, 70, True), (0.0, False, 70, True)])
def test_attention_options_in_large_tiles(D, act, codes, softcap, slopes, window, prefix):
    lengths = [(200, 600), (1, 300), (33, 40)]
    s = torch.exp2(-torch.arange(64, device="cuda").float() / 8) if slopes else None
    first = [37, 37, 40] if prefix else None
    Setup(lengths, kvh=8, D=D, P=32, act=act, codes=codes, window=window, prefix=first, **LARGE).check(
        softcap=softcap, slopes=s, scale=-0.3 if softcap else None)


@pytest.mark.parametrize("D,act,codes", [(128, torch.float16, torch.int8), (64, torch.bfloat16, torch.float8_e4m3fn)])
def test_large_tiles_of_requests_without_keys(D, act, codes):
    """lens 0, fewer tokens than rows, pages outside the pool; more rows than said."""
    s = Setup([(2, 40), (30, 0), (0, 50), (50, 20), (70, 0), (9, 200), (90, 20)], kvh=4, D=D, P=16, act=act, codes=codes, **LARGE)
    dead = [torch.zeros(max(L, 1), dtype=torch.bool) for _, L in s.lengths]
    for r, page, bad in ((0, 1, -1), (5, 0, s.pool), (5, 3, 2 ** 31 - 1), (5, 7, -2 ** 31), (6, 1, -1)):
        s.batch.table[r, page] = bad
        dead[r][16 * page:16 * page + 16] = True
    s.check(dead=dead)
    s.batch.table[5].fill_(s.pool + 5)
    dead[5][:] = True
    s.check(dead=dead)
    Setup([(300, 400), (1, 33), (3, 3)], kvh=8, D=D, P=16, act=act, codes=codes, max_new=40, **LARGE).check()


def test_large_tiles_of_starts_that_contradict_themselves():
    s = Setup([(3, 900), (40, 1200), (1, 2500), (2, 33)], kvh=8, D=128, P=16, act=torch.bfloat16, codes=torch.int8, **LARGE)
    want, T = s.run().clone(), s.batch.tokens
    for starts in ([T, 0, T, 0, T], [-5, 2 ** 31 - 1, 3, -2 ** 31, 50], [T] * 5, [0, T, T, 0, T]):
        s.batch.starts.copy_(_ints(starts))
        s.batch.lens.copy_(_ints([2 ** 31 - 1, 1200, -7, 2 ** 30]))
        s.run()
        s.batch.starts.copy_(_ints(s.starts))
        s.batch.lens.copy_(_ints(s.lens))
        s.out.fill_(9.0)
        assert torch.equal(s.run(), want)


@pytest.mark.parametrize("D,kvh,act,codes", [(128, 1, torch.float16, torch.int8), (64, 2, torch.bfloat16, torch.float8_e4m3fn),
                                             (128, 8, torch.bfloat16, torch.int8)])
def test_large_tiles_in_stretches(D, kvh, act, codes):
    """Few rows of long requests: stretches of a tile, joined in order; strides of other tensors between."""
    s = Setup([(5, 9000), (20, 3000)], kvh=kvh, D=D, P=64, act=act, codes=codes, **LARGE)
    s.check()
    want = s.out.clone()
    T, H, _ = s.q.shape
    packed = torch.full((T, H + 4, D), 3.0, dtype=s.q.dtype, device="cuda")
    packed[:, :H] = s.q
    wide = torch.full((T, H + 1, D), 3.0, dtype=s.q.dtype, device="cuda")
    s.q, s.out = packed[:, :H], wide[:, :H]
    for _ in range(5):
        s.out.fill_(9.0)
        assert torch.equal(s.run(), want) and bool((wide[:, H:] == 3.0).all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("codes", CODES)
@pytest.mark.parametrize("act,size", [(torch.float16, 2.0 ** -24), (torch.float16, 2.0 ** -20), (torch.float16, 2.0 ** -14),
                                      (torch.bfloat16, 2.0 ** -90), (torch.float16, 3e4)])
def test_large_tiles_of_values_at_the_ends_of_the_range(act, codes, size, D):
    s = Setup([(200, 200)], kvh=2, D=D, P=16, act=act, codes=codes, **LARGE)
    g = torch.Generator(device="cuda").manual_seed(3)
    slots = [s.table[0][j // 16] * 16 + j % 16 for j in range(200)]
    k = torch.randn(200, 2, D, device="cuda", generator=g).to(act)
    v = (torch.randn(200, 2, D, device="cuda", generator=g).clamp(-2, 2) * size).to(act)
    s.kv.append(s.cache, k, v, _ints(slots))
    s.check()
    assert bool(torch.isfinite(s.out.float()).all()) and (size < 2.0 ** -20 or bool((s.out != 0).any()))


@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("act,codes", [(torch.float16, torch.int8), (torch.bfloat16, torch.float8_e4m3fn), (torch.float16, torch.float8_e4m3fn)])
@pytest.mark.parametrize("D,prefix,softcap", [(128, None, 0.0), (64, [37, 0, 90, 200], 0.0), (128, [1, 64, 0, 5], 9.0)])
def test_attention_where_no_row_looks_there_may_be_anything(large, act, codes, D, prefix, softcap):
    """Tokens between a prefix and the window: pages whose scales are NaN or infinite, codes that are NaN."""
    lengths, window, P = [(1, 1000), (3, 900), (40, 1200), (100, 700)], 70, 32
    more = LARGE if large else dict(heads=8)
    s = Setup(lengths, kvh=2, D=D, P=P, act=act, codes=codes, window=window, prefix=prefix, **more)
    for r, (n, L) in enumerate(lengths):
        lo, hi = (prefix[r] if prefix else 0), L - n - window + 1
        for j in range(lo, hi):
            page, at = s.table[r][j // P], j % P
            for t in (s.cache.k.view(torch.uint8)[page, :, at], s.cache.v.view(torch.uint8)[page, :, :, at]):
                t.fill_(0x7F if codes is torch.float8_e4m3fn else 0x80)
            if j % P == 0 and j + P <= hi:
                s.cache.k_scale[page] = float("nan") if j // P % 2 else float("inf")
                s.cache.v_scale[page] = float("inf") if j // P % 3 else float("nan")
    s.check(softcap=softcap)


@pytest.mark.parametrize("rows", [1, 17])
def test_attention_of_more_requests_than_threads(rows):
    """A plan of several requests a thread, and of more tiles than threads."""
    rng = random.Random(rows)
    lengths = [(n, n + rng.randrange(0, 90)) for n in (rng.choice((0, 1, rows, rows)) for _ in range(1100))]
    lengths[700] = (rows, 4000)
    Setup(lengths, 2, 2, 64, 32, torch.bfloat16, torch.int8, pad=3).check()


@pytest.mark.parametrize("lengths", [[(1, 3000)] * 3, [(128, 900), (1, 50)]])
def test_attention_is_repeatable(lengths):
    s = Setup(lengths, 8, 1, 128, 64, torch.bfloat16, torch.int8)
    first = s.run().clone()
    for _ in range(10):
        s.out.fill_(9.0)
        assert torch.equal(s.run(), first)


def test_attention_past_32_bits():
    """A cache of more than 2^32 bytes, pages at its far end."""
    kv, P, D, kvh = _kv(), 128, 128, 8
    pages = (1 << 32) // (P * D * kvh) + 40
    cache = kv.new_cache(pages, kvh, P, D, torch.bfloat16)
    small = _random_cache(kv, 8, kvh, P, D, torch.bfloat16, torch.int8, 2)
    order = [pages - 1 - 3 * i for i in range(8)]
    for i, p in enumerate(order):
        for big, little in zip(cache.tensors(), small.tensors()):
            big[p] = little[i]
    for lengths in ([(1, 1000)], [(40, 1000)]):
        q = torch.randn(lengths[0][0], 16, D, device="cuda").to(torch.bfloat16)
        outs = []
        for c, row in ((small, list(range(8))), (cache, order)):
            b = kv.Batch(_ints([row]), q.shape[0], starts=_ints([0, q.shape[0]]), lens=_ints([1000]))
            plan = kv.AttentionPlan(c, b, 16)
            ws = torch.zeros(kv.attention_workspace(plan), dtype=torch.uint8, device="cuda")
            kv.attention_plan(plan)
            outs.append(kv.attention(plan, q, torch.empty_like(q), workspace=ws))
        assert torch.equal(*outs)
    # and written and read there
    x = torch.randn(3, kvh, D, device="cuda").to(torch.bfloat16)
    slots = _ints([(pages - 2) * P + 5, (pages - 2) * P + 6, (pages - 5) * P])
    a, b = torch.empty_like(x), torch.empty_like(x)
    kv.append(cache, x, x, slots)
    kv.read(cache, slots, a, b)
    assert torch.equal(a, b) and float((a - x).float().norm() / x.float().norm()) < 0.02


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

class Server:
    """A small serving loop: a pool, two layers' caches, requests that grow."""

    def __init__(self, R, T, max_new, heads=8, kvh=2, D=64, P=16, act=torch.bfloat16, codes=torch.int8, width=40):
        kv = self.kv = _kv()
        self.R, self.T, self.P, self.act = R, T, P, act
        self.table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
        self.batch = kv.Batch(self.table, T, max_new=max_new)
        self.held, self.fresh = _ints([0] * R), _ints([0] * R)
        self.free = torch.randperm(R * width, device="cuda").to(torch.int32)
        self.slots, self.positions, self.taken = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (T, T, 2))
        self.caches = [kv.new_cache(R * width, kvh, P, D, act, codes) for _ in range(2)]
        self.rope = _rope(kv, D, False)
        self.plan = kv.AttentionPlan(self.caches[0], self.batch, heads)
        self.ws = torch.zeros(kv.attention_workspace(self.plan), dtype=torch.uint8, device="cuda")
        self.x = [tuple(torch.zeros(T, h, D, dtype=act, device="cuda") for h in (heads, kvh, kvh)) for _ in range(2)]
        self.qr = [torch.zeros_like(x[0]) for x in self.x]
        self.out = [torch.full_like(x[0], 9.0) for x in self.x]

    def step(self, stream=None):
        kv = self.kv
        kv.pages(self.batch, self.held, self.fresh, self.free, self.slots, self.positions, self.taken,
                 page_tokens=self.P, stream=stream)
        kv.attention_plan(self.plan, stream=stream)
        for cache, (q, k, v), qr, out in zip(self.caches, self.x, self.qr, self.out):
            kv.append(cache, k, v, self.slots, self.positions, rope=self.rope, q=q, q_out=qr, stream=stream)
            kv.attention(self.plan, qr, out, workspace=self.ws, cache=cache, stream=stream)

    def feed(self, fresh, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.fresh.copy_(_ints(fresh))
        for group in self.x:
            for t in group:
                t.copy_(torch.randn(t.shape, device="cuda", generator=g))
        for o in self.out:
            o.fill_(9.0)

    def advance(self):
        n = int(self.taken[0])
        self.free[:self.free.numel() - n] = self.free[n:].clone()
        self.held += self.fresh

    def check(self):
        kv = self.kv
        starts, lens = self.batch.starts.tolist(), self.batch.lens.tolist()
        for cache, qr, out in zip(self.caches, self.qr, self.out):
            k, v = [], []
            for r, L in enumerate(lens):
                slots = [int(self.table[r, j // self.P]) * self.P + j % self.P for j in range(L)]
                a, b = (torch.empty(max(L, 1), cache.kv_heads, cache.head_dim, dtype=self.act, device="cuda") for _ in range(2))
                kv.read(cache, _ints(slots), a[:L], b[:L])
                k.append(a[:L].cpu().double())
                v.append(b[:L].cpu().double())
            want, bound = U.plain_attention(qr.cpu(), k, v, starts, lens, qr.shape[1], scale=cache.head_dim ** -0.5)
            got, end = out.cpu().double(), starts[-1]
            assert bool(((got - want).abs() <= bound)[:end].all())
            assert bool((got[end:] == 9.0).all())


def test_a_run_of_steps():
    """Prompts in chunks beside decoding requests, two layers, every step against the plain reference."""
    s = Server(5, 200, 120)
    for i, fresh in enumerate(([120, 30, 1, 0, 0], [60, 1, 1, 0, 17], [1, 1, 1, 100, 1], [1, 1, 1, 1, 1], [1, 0, 1, 1, 1])):
        s.feed(fresh, i)
        s.step()
        s.check()
        s.advance()
    assert s.held.tolist() == [183, 33, 5, 102, 20]


def test_a_captured_step_serves_other_lengths():
    """One graph of a decoding step, replayed as the requests grow and come and go, with eager work and
    waits between; each replay against the reference; a second graph shares its workspace."""
    s, other = Server(4, 4, 1, heads=16, kvh=1, width=100), Server(3, 150, 64, heads=16, kvh=1, width=100)
    small = s if s.ws.numel() >= other.ws.numel() else other
    s.ws = other.ws = small.ws
    graphs = []
    for x in (s, other):
        x.feed([1] * x.R, 0)
        x.step()
        torch.cuda.synchronize()
        x.batch.lens.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            x.step()
        graphs.append(graph)
    for i in range(6):
        for x, graph, fresh in ((s, graphs[0], [1, i % 2, 1, 1]), (other, graphs[1], [64 - i, 1, 30 if i else 0])):
            x.feed(fresh, 10 + i)
            if i == 3:
                x.held[0] = 1500 - (1500 % x.P)  # far into the request: pages that hold what they hold
                x.table[0, :1500 // x.P] = torch.arange(1500 // x.P, device="cuda")
            graph.replay()
            torch.cuda.synchronize()
            x.check()
            x.advance()
            torch.randn(1000, device="cuda").sum().item()


def test_calls_of_unlike_sizes_share_a_workspace():
    """Stretches joined by both kernels, of other head counts and batches, one workspace in turn: what one
    call leaves there is nothing to the next."""
    act, codes = torch.bfloat16, torch.int8
    setups = [Setup([(1, 5000)], 16, 1, 64, 64, act, codes), Setup([(70, 3000), (1, 2000)], 16, 2, 128, 64, act, codes),
              Setup([(1, 4000)] * 3, 8, 4, 128, 64, act, codes), Setup([(300, 2500)], 4, 4, 64, 64, act, codes)]
    ws = max((s.ws for s in setups), key=torch.Tensor.numel)
    want = []
    for s in setups:
        s.check()
        want.append(s.out.clone())
        s.ws = ws
    ws.zero_()
    for order in ([0, 1, 2, 3], [3, 0, 1], [2, 1, 0], [1, 1, 3, 0]):
        for i in order:
            setups[i].out.fill_(9.0)
            assert torch.equal(setups[i].run(), want[i]), i


def test_other_streams():
    s = Server(3, 90, 40)
    stream = torch.cuda.Stream()
    s.feed([40, 1, 7], 3)
    torch.cuda.synchronize()
    s.step(stream)
    stream.synchronize()
    s.check()
    a, b = [Server(3, 90, 40) for _ in range(2)]  # two at once, a workspace each
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, x in enumerate((a, b)):
        x.feed([40, 2, 9], i)
    torch.cuda.synchronize()
    for _ in range(3):
        for x, st in zip((a, b), streams):
            x.step(st)
    torch.cuda.synchronize()
    a.check()
    b.check()
