"""The cache's operators and attention at the far ends of their stated ranges, on
the GPU, against formulas in 64 bits."""
from __future__ import annotations

import math

import pytest
import torch

import kv_util as U
from test_gpu_kv import ACTS, CODES, LARGE, Setup, _ints, _kv

pytestmark = pytest.mark.gpu

# the least power of two whose multiple by the largest code passes the activation type's end
LAST_SCALE = {(torch.float16, torch.int8): 2.0 ** 10, (torch.bfloat16, torch.int8): 2.0 ** 122,
              (torch.float16, torch.float8_e4m3fn): 2.0 ** 8, (torch.bfloat16, torch.float8_e4m3fn): 2.0 ** 120}


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("codes", CODES)
@pytest.mark.parametrize("P,D,off", [(16, 64, 1), (16, 128, 4), (32, 64, 7), (128, 128, 66)])
def test_scales_that_grow_past_the_types_end(act, codes, P, D, off):
    """The largest codes of the last scale but one, then the type's largest value in the same page: no code,
    old or new, stands for a value past the type's largest (INT8: 127 / 2 is held to 63)."""
    kv = _kv()
    last, top = LAST_SCALE[act, codes], float(torch.finfo(act).max)
    cache = kv.new_cache(3, 2, P, D, act, codes)
    # places 0..off-1 at half the last scale: its largest code (either sign), and smaller ones
    x = torch.randint(-127, 128, (off, 2, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(P)).double()
    x[:, :, 0], x[:, :, 1], x[:, :, 2], x[:, :, D - 1] = 127, -127, 126, 127
    if codes is torch.float8_e4m3fn:
        x = U.nearest(x.cpu() * 448 / 127, codes).cuda()
    old = (x * (last / 2)).to(act)
    assert torch.equal(old.double(), x * (last / 2)) and bool(torch.isfinite(old).all())
    kv.append(cache, old, old.clone(), _ints([P + i for i in range(off)]))
    assert cache.k_scale[1].tolist() == [last / 2] * 2 and cache.v_scale[1].tolist() == [last / 2] * 2
    new = torch.zeros(1, 2, D, dtype=act, device="cuda")
    new[:, :, 5], new[:, :, 6] = top, -top
    kv.append(cache, new, new.clone(), _ints([P + off]))
    assert cache.k_scale[1].tolist() == [last] * 2 and cache.v_scale[1].tolist() == [last] * 2
    most = U.top_code(last, codes, act)
    want = torch.cat([U.nearest(x.cpu() / 2, codes).clamp(-most, most), (new.cpu().double() / last).clamp(-most, most)]) * last
    ko, vo = (torch.empty(off + 1, 2, D, dtype=act, device="cuda") for _ in range(2))
    kv.read(cache, _ints([P + i for i in range(off + 1)]), ko, vo)
    for got in (ko, vo):
        assert bool(torch.isfinite(got).all())
        assert torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("codes", CODES)
@pytest.mark.parametrize("lengths,more", [([(1, 200)], {}), ([(20, 200)], {}), ([(200, 200)], LARGE)])
def test_attention_over_scales_that_grew_past_the_types_end(codes, lengths, more):
    """Values of fp16's whole range, written so that pages' scales grow to the last one: outputs are finite, also of
    rows whose weight for such a token is zero."""
    act, L = torch.float16, lengths[0][1]
    s = Setup(lengths, kvh=2, D=64, P=16, act=act, codes=codes, **{"heads": 4, **more})
    g = torch.Generator(device="cuda").manual_seed(1)
    last = LAST_SCALE[act, codes]
    k = torch.randn(L, 2, 64, device="cuda", generator=g).to(act)
    v = (torch.randint(-1, 2, (L, 2, 64), device="cuda", generator=g) * U.TOP[codes] * last / 2).to(act)
    v[15::16, :, 3::7] = float(torch.finfo(act).max)
    slots = [s.table[0][j // 16] * 16 + j % 16 for j in range(L)]
    old = [j for j in range(L) if j % 16 != 15]
    rest = [j for j in range(L) if j % 16 == 15]
    for part in (old, rest):  # (the last place of a page comes after the others)
        s.kv.append(s.cache, k[part], v[part], _ints([slots[j] for j in part]))
    assert float(s.cache.v_scale[s.table[0][0]].max()) == last
    for scale in (None, 40.0):  # (and weights that are zero but for one token)
        s.check(scale=scale)
        assert bool(torch.isfinite(s.out[:lengths[0][0]]).all())


@pytest.mark.parametrize("D,act,codes", [(64, torch.float16, torch.int8), (128, torch.bfloat16, torch.float8_e4m3fn)])
@pytest.mark.parametrize("lengths,more", [([(1, 700), (2, 90)], dict(heads=4)), ([(20, 300), (7, 7)], dict(heads=8)),
                                          ([(200, 300), (1, 50)], LARGE)])
def test_caps_of_any_size(D, act, codes, lengths, more):
    """Scores far below the cap (which then makes no difference), about it, far above it; caps whose reciprocal
    is not a float, or is not a normal one."""
    s = Setup(lengths, kvh=2, D=D, P=32, act=act, codes=codes, **more)
    for cap in (3e38, 1e30, 1e8, 1e6, 1e4, 300.0, 20.0, 1.0, 1e-3, 1e-30, 1e-39, 1e-45):
        s.check(softcap=cap, scale=0.3)
    s.check(softcap=1e7, scale=-2.0)


def test_caps_where_weights_are_even():
    """Scores of at most 1 that a cap of 10^8 leaves as they are: the weights follow them."""
    act = torch.float16
    s = Setup([(1, 64)], 1, 1, 64, 16, act, torch.int8)
    g = torch.Generator(device="cuda").manual_seed(4)
    slots = _ints([s.table[0][j // 16] * 16 + j % 16 for j in range(64)])
    k = torch.zeros(64, 1, 64, dtype=act, device="cuda")
    k[:, 0, 0] = torch.linspace(-1, 1, 64, device="cuda").to(act)
    v = torch.randn(64, 1, 64, device="cuda", generator=g).to(act)
    s.kv.append(s.cache, k, v, slots)
    s.q.zero_()
    s.q[:, :, 0] = 1.0
    for cap in (1e3, 1e5, 1e8, 3e38):
        s.check(scale=1.0, softcap=cap)


# ---------------------------------------------------------------------------
# plans of the longest requests: written, and only their shares counted; attention over them would take hours
# ---------------------------------------------------------------------------

def _plan_in_margins(kv, plan, margin=1 << 16):
    """The plan's own bytes after a call, which stand between margins that have to stay as they are."""
    n = plan.buffer.numel()
    room = torch.full((margin + n + 16 * margin,), 0x5A, dtype=torch.uint8, device="cuda")
    at = room[margin:margin + n]
    plan.c.plan = at.data_ptr()
    kv.attention_plan(plan)
    torch.cuda.synchronize()
    assert bool((room[:margin] == 0x5A).all()) and bool((room[margin + n:] == 0x5A).all())
    return at.view(torch.int32).view(-1, 16).cpu()  # a share is 64 bytes: its sizes' number (0: none), its request, ...


def test_plans_of_the_longest_requests_in_tiles():
    """8192 tiles of 2^24 steps: a stretch's length passes 31 bits before it is held to a request's steps."""
    kv = _kv()
    T, P, width = 131072, 128, 1 << 23
    cache = kv.new_cache(1, 8, P, 64, torch.float16)
    batch = kv.Batch(torch.empty((1, width), dtype=torch.int32, device="cuda"), T, starts=_ints([0, T]), lens=_ints([2 ** 30 - 1]))
    plan = kv.AttentionPlan(cache, batch, 64)
    tiles = T * 8 // 128
    shares = _plan_in_margins(kv, plan)
    shares = shares[shares[:, 0] != 0]
    assert shares.shape[0] == tiles and bool((shares[:, 1] == 0).all())  # one stretch each
    # what a length out of bounds gives
    for bad in (2 ** 31 - 1, 2 ** 30, -1):
        batch.lens.fill_(bad)
        _plan_in_margins(kv, plan)


def test_plans_of_the_longest_requests_of_few_rows():
    """160 requests of 2^24 steps and 512 kv heads, one stretch wanted in all: 2.7 10^9 steps."""
    kv = _kv()
    R, P, width = 160, 128, 1 << 23
    cache = kv.new_cache(1, 512, P, 64, torch.float16)
    table = torch.empty((R, width), dtype=torch.int32, device="cuda")
    batch = kv.Batch(table, R, max_new=1, starts=_ints(list(range(R + 1))), lens=_ints([2 ** 30 - 1] * R))
    shares = _plan_in_margins(kv, kv.AttentionPlan(cache, batch, 512))
    shares = shares[shares[:, 0] != 0]
    assert sorted(shares[:, 1].tolist()) == list(range(R))  # one stretch each


# ---------------------------------------------------------------------------
# contradicting arrays
# ---------------------------------------------------------------------------

def _between_margins(n, dtype, rows=1 << 16):
    """(all, the n elements in the middle): the rest is a pattern."""
    room = torch.full((n + 2 * rows,), 0x5A, dtype=torch.uint8, device="cuda") if dtype is torch.uint8 else \
        torch.full((n + 2 * rows,), 5.0, dtype=dtype, device="cuda")
    return room, room[rows:rows + n], rows


@pytest.mark.parametrize("kvh,more", [(1, dict(heads=8, pad=4, D=64)), (8, dict(D=128, **LARGE))])
def test_contradicting_starts_touch_nothing_else(kvh, more):
    """Out, plan and workspace between margins that stay as they are, whatever starts and lens hold; rows behind the
    step's tokens and the inputs too; and a call after it is right."""
    s = Setup([(3, 900), (40, 1200), (1, 2500), (2, 33)], kvh=kvh, P=16, act=torch.bfloat16, codes=torch.int8, **more)
    want, T = s.run().clone(), s.batch.tokens
    rooms = []
    for name, t in (("out", s.out), ("plan", s.plan.buffer), ("ws", s.ws)):
        room, middle, rows = _between_margins(t.numel(), t.dtype)
        rooms.append((name, room, rows, t.numel()))
        if name == "out":
            s.out = middle.view(t.shape)
        elif name == "plan":
            s.plan.buffer, s.plan.c.plan = middle, middle.data_ptr()
        else:
            middle.zero_()
            s.ws = middle
    kept = [t.clone() for t in (*s.cache.tensors(), s.q, s.batch.table)]
    n = s.starts[-1]
    for starts in ([n, 0, n, 0, n], [-5, 2 ** 31 - 1, 3, -2 ** 31, 50], [n] * 5, [0, n, n, 0, n], [T, 0, T, 0, T], [9, 3, 1, 0, -1]):
        for lens in ([2 ** 31 - 1, 1200, -7, 2 ** 30], [0, 0, 0, 0], [900, 1200, 2500, 33]):
            s.batch.starts.copy_(_ints(starts))
            s.batch.lens.copy_(_ints(lens))
            s.run()
            s.batch.starts.copy_(_ints(s.starts))
            s.batch.lens.copy_(_ints(s.lens))
            s.out.fill_(9.0)
            assert torch.equal(s.run(), want)
            for name, room, rows, size in rooms:
                fill = 0x5A if room.dtype is torch.uint8 else 5.0
                assert bool((room[:rows] == fill).all()) and bool((room[rows + size:] == fill).all()), (name, starts, lens)
    for before, t in zip(kept, (*s.cache.tensors(), s.q, s.batch.table)):
        assert torch.equal(before.view(torch.uint8), t.view(torch.uint8))


# ---------------------------------------------------------------------------
# pages outside the pool, in steps that every row would see whole
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("codes", CODES)
@pytest.mark.parametrize("D,P", [(64, 16), (128, 32), (128, 64), (64, 128)])
@pytest.mark.parametrize("options", [{}, dict(softcap=7.0, slopes=True)])
@pytest.mark.parametrize("lengths,more", [([(1, 1500), (2, 700)], dict(heads=4)), ([(20, 1500), (9, 700)], dict(heads=8)),
                                          ([(200, 1500), (90, 700)], LARGE)])
def test_pages_outside_the_pool(act, codes, D, P, options, lengths, more):
    """One page in a step, the first, the last that is whole, several in a row; what stands at the pool's first page,
    which a kernel may read in their place, is no number."""
    s = Setup(lengths, kvh=2, D=D, P=P, act=act, codes=codes, **more)
    kinds = (-1, s.pool, 2 ** 31 - 1, -2 ** 31)
    dead = [torch.zeros(L, dtype=torch.bool) for _, L in lengths]
    for r, (n, L) in enumerate(lengths):
        last = (L - n) // P - 1  # every row sees the whole of it
        for x, page in enumerate((0, 2, last // 2, last // 2 + 1, last // 2 + 2, last)):
            s.batch.table[r, page] = kinds[x % 4]
            dead[r][P * page:P * page + P] = True
        for page in range(-(-L // P)):  # pages of the pool's first place go too
            if s.table[r][page] == 0:
                s.batch.table[r, page] = -1
                dead[r][P * page:P * page + P] = True
    for scale in (s.cache.k_scale, s.cache.v_scale):
        scale[0] = float("nan")
    s.cache.v.view(torch.uint8)[0] = 0x7F
    slopes = torch.exp2(-torch.arange(s.heads, device="cuda").float() / 8) if options.get("slopes") else None
    s.check(softcap=options.get("softcap", 0.0), slopes=slopes, dead=dead)


# ---------------------------------------------------------------------------
# weights far below the largest
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("act,codes", [(torch.float16, torch.int8), (torch.float16, torch.float8_e4m3fn), (torch.bfloat16, torch.int8)])
@pytest.mark.parametrize("lengths,more", [([(1, 60000)], dict(heads=4)), ([(20, 9000)], dict(heads=8)), ([(1600, 3000)], LARGE)])
@pytest.mark.parametrize("D,power", [(64, 20.0), (128, 25.3), (64, 26.2)])
def test_weights_far_below_the_largest(act, codes, lengths, more, D, power):
    """A first token of weight 1 and value 0, all others of weight 2^-power and value 1: together they are what
    comes out, though each is near or below the least number of fp16."""
    n, L = lengths[0]
    s = Setup(lengths, kvh=2, D=D, P=64, act=act, codes=codes, **more)
    slots = [s.table[0][j // 64] * 64 + j % 64 for j in range(L)]
    k = torch.zeros(L, 2, D, dtype=act, device="cuda")
    k[1:, :, 0] = -1.0
    v = torch.ones(L, 2, D, dtype=act, device="cuda")
    v[0] = 0.0
    s.kv.append(s.cache, k, v, _ints(slots))
    s.q.zero_()
    s.q[:, :, 0] = 1.0
    scale = power * math.log(2)
    got = s.run(scale=scale)[:n].cpu().double()
    others = torch.arange(L - n, L).double() * math.exp(-float(torch.tensor(scale, dtype=torch.float32)))
    want = (others / (1 + others))[:, None, None].expand_as(got)
    # Of the weight of each: its rounding (half a step, or in fp16 half of its least number, 2^-25, to a largest
    # weight of 2^3 at least), and its score's, a product and three roundings of a number of `power` in fp32: 2^-22 power.
    # Of the sum over them as much, and L roundings of the sums at 2^-24 each; and that of the output.
    u = U.U[act]
    each = torch.maximum(torch.tensor(u), torch.tensor(2.0 ** (power - 28) if act is torch.float16 else 0.0)).double()
    bound = want * (2 * each + 2.0 ** -22 * power + L * 2.0 ** -24 + u) + (2.0 ** -25 if act is torch.float16 else 0.0)
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / want).max())


@pytest.mark.parametrize("heads,kvh", [(1024, 1024), (1024, 512), (1024, 32), (1024, 1), (512, 512)])
def test_the_most_heads(heads, kvh):
    """More kv heads than stretches are wanted, and groups of a thousand heads."""
    Setup([(1, 70), (2, 33)], heads, kvh, 64, 16, torch.float16, torch.int8, pad=1).check()
    Setup([(20, 50), (1, 300)], heads, kvh, 64, 32, torch.bfloat16, torch.float8_e4m3fn).check()
