"""GPU parity of the adapters of many requests against the float64 oracle:
slots, ranks, ids, strides and values where they can go wrong, the layer's
paths they join, grouped calls, and replays of a captured graph."""
from __future__ import annotations

import contextlib

import numpy as np
import pytest
import torch

from oracle import spear_oracle as O
from paper_2606_11244_amd import synth as S

from gpu_util import assert_parity, log

pytestmark = pytest.mark.gpu

DT = {S.F16: torch.float16, S.BF16: torch.bfloat16}
# half a step of the activation dtype, relative; what a factor held as the sum
# of two such numbers may be off, relative
HALF = {S.F16: 2.0 ** -11, S.BF16: 2.0 ** -8}
SPLIT = {S.F16: 2.0 ** -21, S.BF16: 2.0 ** -15}
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class Slots:
    """Adapters of L slots for M tokens, on the GPU; NaN lies wherever nothing
    may be read: past each slot's rank and between strided slots."""

    def __init__(self, M, N, K, L, R, dt, *, ids="random", mixed=False, scale=True, gap=0, seed=0):
        g = torch.Generator().manual_seed(seed * 7919 + M * 31 + N)
        t = DT[dt]
        self.M, self.N, self.K, self.dt = M, N, K, dt
        self.ranks = None
        if mixed:
            self.ranks = torch.randint(0, R + 2, (L,), generator=g, dtype=torch.int32)  # R + 1: all of R
            self.ranks[0] = R
        A = torch.randn(L, R, K, generator=g) * 0.05
        B = torch.randn(L, N, R, generator=g) * 0.05
        for a in range(L):
            n = R if self.ranks is None else min(int(self.ranks[a]), R)
            A[a, n:], B[a, :, n:] = NAN, NAN
        self.A, self.B = self._spread(A.to(t), gap), self._spread(B.to(t), gap)
        self.scale = (0.5 + torch.rand(L, generator=g)) if scale else None
        if ids == "random":
            i = torch.randint(-1, L + 1, (M,), generator=g, dtype=torch.int32)
        elif ids == "runs":
            i = (torch.arange(M) * L // max(M, 1)).to(torch.int32)
        elif ids == "one":
            i = torch.full((M,), L - 1, dtype=torch.int32)
        elif ids == "none":
            i = torch.where(torch.arange(M) % 2 == 0, -7, 2 ** 31 - 1).to(torch.int32)
        else:  # in turn
            i = (torch.arange(M) % L).to(torch.int32)
        self.ids = i

    @staticmethod
    def _spread(T, gap):
        if not gap:
            return T
        flat = torch.full((T.shape[0], T[0].numel() + gap), NAN, dtype=T.dtype)
        flat[:, :T[0].numel()] = T.reshape(T.shape[0], -1)
        return flat[:, :T[0].numel()].view(T.shape)

    def device(self):
        from paper_2606_11244_amd import spear as sp

        def cu(t):
            if t is None or t.is_contiguous():
                return None if t is None else t.cuda()
            return t.as_strided((t.untyped_storage().nbytes() // t.element_size(),), (1,)).cuda().as_strided(t.shape, t.stride())
        return sp.adapters(cu(self.A), cu(self.B), cu(self.ids), ranks=cu(self.ranks), scale=cu(self.scale))

    def term(self, x):
        A, B = torch.nan_to_num(self.A.double()).numpy(), torch.nan_to_num(self.B.double()).numpy()
        return O.adapters_term(x, A, B, self.ids.numpy(), self.ranks, self.scale)

    def bound(self, x, term, y):
        """|error| of y, elementwise: the fp32 sums over K and then over the
        ranks, worst case (one rounding of 2^-24 a step, of sums of magnitudes),
        the coordinates held in two parts, and two roundings to the activation
        dtype, of the term with the residual and of y."""
        A, B = (torch.nan_to_num(v.double()).abs().numpy() for v in (self.A, self.B))
        mag = O.adapters_term(np.abs(x), A, B, self.ids.numpy(), self.ranks, self.scale)
        steps = (self.K + A.shape[1] + 4) * 2.0 ** -24 + SPLIT[self.dt]
        tiny = 2.0 ** -24 if self.dt == S.F16 else 0.0  # a step of a subnormal
        return steps * mag + HALF[self.dt] * 1.001 * (np.abs(term) + np.abs(y)) + tiny


def _layer(M, N, K, dt, seed=0, **kw):
    from paper_2606_11244_amd import spear as sp
    L = S.make_layer(M=M, N=N, K=K, group_size=128, act_dtype=dt, seed=seed, **dict(dict(rank=0), **kw))
    return L, sp.DeviceLayer(L)


def _x(dl):
    return dl.x.double().cpu().numpy()


def _call(dl, ad, ws=None, ec=False, y=None, **kw):
    from paper_2606_11244_amd import spear as sp
    m = dl.member(dl.problem(), with_ec=ec)
    if ws is None:
        n = sp.adapters_workspace([dict(m, adapters=ad)])
        ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
        ws[(128 + 1024) * 1024:] = 255  # the data regions need no clearing: every byte NaN
    y = dl.y if y is None else y
    sp.w4ec_linear_adapters(m["prob"], dl.x, dl.qweight, dl.scales, dl.zeros, ad, y,
                            ec_args=m["ec_args"], workspace=ws, **kw)
    torch.cuda.synchronize()
    return y.double().cpu().numpy()


# (M, N, K, L, R, options): token counts around the tiles, rows around 16, 64
# and 128, every kind of rank, one slot to more slots than tokens
SHAPES = [
    (1, 16, 128, 1, 8, dict(ids="one")), (1, 520, 1152, 9, 16, dict(ids="turn")),
    (2, 129, 256, 3, 1, {}), (3, 64, 128, 2, 4, dict(mixed=True)), (5, 1000, 512, 7, 13, dict(mixed=True)),
    (8, 1, 128, 4, 16, dict(ids="turn")), (16, 256, 1024, 16, 16, dict(ids="turn")),
    (17, 272, 384, 5, 24, dict(gap=8)), (16, 4104, 256, 3, 8, dict(scale=False)),
    (31, 40, 640, 40, 40, dict(ids="turn", mixed=True)), (33, 200, 256, 2, 64, dict(ids="runs")),
    (48, 520, 1024, 64, 64, dict(mixed=True)), (64, 130, 2048, 30, 32, dict(ids="turn")),
    (65, 136, 256, 4, 100, dict(gap=24)), (70, 24, 128, 70, 7, dict(ids="turn")),
    (127, 1024, 512, 6, 16, dict(ids="runs")), (130, 300, 1152, 33, 48, dict(mixed=True)),
    (257, 144, 256, 3, 256, dict(ids="runs")), (300, 514, 384, 300, 5, dict(ids="turn")),
    (520, 640, 512, 9, 128, dict(ids="runs", mixed=True)), (1030, 72, 128, 5, 16, dict(ids="random")),
    (40, 64, 256, 3, 16, dict(ids="none")), (9, 33, 14336, 4, 32, dict(ids="turn")),
    (12, 7000, 128, 5, 20, {}), (100, 8, 8192, 8, 16, dict(ids="turn")),
    (128, 520, 1152, 40, 24, dict(ids="turn", mixed=True)), (128, 1000, 256, 2, 72, dict(ids="runs")),
    (129, 264, 512, 5, 16, dict(ids="runs")),
]


@pytest.mark.parametrize("M,N,K,L,R,opt", SHAPES)
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
def test_term_alone(M, N, K, L, R, opt, dt):
    """Scales of zero: the product is exactly zero, y is the term."""
    log(f"adapters M={M} N={N} K={K} L={L} R={R} {opt} dt={dt}")
    _, dl = _layer(M, N, K, dt, seed=M + N)
    dl.scales.zero_()
    s = Slots(M, N, K, L, R, dt, seed=R, **opt)
    buf = torch.full((M + 2, N), 7.0, dtype=DT[dt], device="cuda")
    y = _call(dl, s.device(), y=buf[:M])
    assert torch.all(buf[M:] == 7.0)  # rows behind the last token
    ref = s.term(_x(dl))
    err, lim = np.abs(y - ref), s.bound(_x(dl), ref, ref)
    assert np.all(err <= lim), (err.max(), (err / lim.clip(1e-30)).max())
    out = (s.ids < 0) | (s.ids >= L)
    assert not y[out.numpy()].any()


@pytest.mark.parametrize("M,N,K,rank", [(4, 512, 1024, 16), (9, 1000, 4096, 48), (48, 520, 1024, 32), (77, 1000, 1408, 24),
                                        (128, 264, 2048, 32), (200, 520, 1024, 16)])
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
@pytest.mark.parametrize("int8,gate", [(True, S.GATE_SIGMOID_LINEAR), (False, S.GATE_TANH_MLP), (True, S.GATE_TANH_MLP)])
def test_beside_other_compensators(M, N, K, rank, dt, int8, gate):
    """INT8 factors and the tanh-MLP gate, on decode and prefill paths."""
    L, dl = _layer(M, N, K, dt, seed=M, rank=rank, ab_int8=int8, gate_kind=gate)
    s = Slots(M, N, K, 7, 16, dt, seed=9, mixed=True)
    log(f"adapters beside M={M} N={N} K={K} rank={rank} dt={dt} int8={int8} gate={gate}")
    assert_parity(_call(dl, s.device(), ec=True), O.w4ec_linear(L) + s.term(_x(dl)), "with adapters")


@contextlib.contextmanager
def in_the_gemm(roles=3):
    """Every call above 64 tokens without an EC on tiles of 256 tokens (by 128 rows:
    roles 2, by 256: roles 3), whose GEMM forms the term itself above 128 tokens."""
    from paper_2606_11244_amd import spear as sp
    sp.set_gemm_tile(256)
    sp.set_gemm_slices(1)
    sp.set_gemm_roles(roles)
    try:
        yield
    finally:
        sp.set_gemm_roles(0)
        sp.set_gemm_slices(0)
        sp.set_gemm_tile(0)


TILED = [s for s in SHAPES if s[0] > 64] + [(135, 264, 384, 5, 20, dict(ids="turn")), (190, 129, 128, 90, 7, dict(mixed=True)),
    (513, 300, 256, 6, 64, dict(ids="turn")), (256, 256, 128, 1, 16, dict(ids="one")), (300, 520, 384, 3, 72, dict(gap=3 * 8)),
    (270, 250, 128, 20, 130, dict(ids="runs", mixed=True)), (700, 257, 256, 4, 65, dict(ids="runs", scale=False)),
    (260, 512, 128, 2, 16, dict(ids="none"))]


@pytest.mark.parametrize("M,N,K,L,R,opt", TILED)
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
@pytest.mark.parametrize("roles", [2, 3])
def test_term_in_the_gemm(M, N, K, L, R, opt, dt, roles):
    log(f"adapters in the GEMM roles={roles} M={M} N={N} K={K} L={L} R={R} {opt} dt={dt}")
    _, dl = _layer(M, N, K, dt, seed=M + N)
    dl.scales.zero_()
    s = Slots(M, N, K, L, R, dt, seed=R, **opt)
    buf = torch.full((M + 2, N), 7.0, dtype=DT[dt], device="cuda")
    res = torch.randn(M, N, generator=torch.Generator().manual_seed(3)).to(DT[dt])
    with in_the_gemm(roles):
        ad = s.device()
        y = _call(dl, ad, y=buf[:M])
        assert torch.all(buf[M:] == 7.0)
        yr = _call(dl, ad, residual=res.cuda())
        inplace = res.cuda()
        assert np.array_equal(_call(dl, ad, y=inplace, residual=inplace), yr)
    x, ref = _x(dl), s.term(_x(dl))
    err, lim = np.abs(y - ref), s.bound(x, ref, ref)
    assert np.all(err <= lim), (err.max(), (err / lim.clip(1e-30)).max())
    assert not y[((s.ids < 0) | (s.ids >= L)).numpy()].any()
    ref = ref + res.double().numpy()
    assert np.all(np.abs(yr - ref) <= s.bound(x, ref, ref))


@pytest.mark.parametrize("M,N,K", [(2049, 8200, 256), (4100, 4104, 128), (1025, 8200, 256)])
def test_large_tiles_by_themselves(M, N, K):
    """The GEMM that AUTO takes there, on sampled tokens."""
    L, R, dt = 5, 24, S.F16
    lay, dl = _layer(M, N, K, dt, seed=7)
    s = Slots(M, N, K, L, R, dt, ids="runs", mixed=True, seed=8)
    y = _call(dl, s.device())
    rows = np.unique(np.linspace(0, M - 1, 60).astype(int))
    x = _x(dl)[rows]
    W = O.dequant(lay.qweight, lay.scales, lay.zeros, lay.group_size)
    s.ids = s.ids[rows]
    assert_parity(y[rows], O.w4_linear(x, W) + s.term(x), "large tiles")


@pytest.mark.parametrize("M,N,K,R", [(4, 520, 512, 16), (40, 264, 1024, 24), (130, 1000, 256, 8)])
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
def test_residual_and_norm(M, N, K, R, dt):
    _, dl = _layer(M, N, K, dt, seed=5)
    dl.scales.zero_()
    s = Slots(M, N, K, 6, R, dt, seed=2)
    res = torch.randn(M, N, generator=torch.Generator().manual_seed(3)).to(DT[dt])
    nw = (1 + 0.1 * torch.randn(N, generator=torch.Generator().manual_seed(4))).to(DT[dt])
    yn = torch.empty(M, N, dtype=DT[dt], device="cuda")
    log(f"adapters tail M={M} N={N} dt={dt}")
    y = _call(dl, s.device(), residual=res.cuda(), norm_w=nw.cuda(), y_norm=yn)
    term = s.term(_x(dl))
    ref = term + res.double().numpy()
    assert np.all(np.abs(y - ref) <= s.bound(_x(dl), ref, ref))
    # the norm is of the stored row: half a step of it, and fp32 sums of N squares
    want = O.rms_norm(y, nw.double().numpy(), 1e-5)
    assert np.all(np.abs(yn.double().cpu().numpy() - want) <= (HALF[dt] * 1.001 + N * 2.0 ** -24) * np.abs(want) + 1e-7)
    # in place: the residual stream is y itself
    y2 = res.cuda()
    got = _call(dl, s.device(), y=y2, residual=y2)
    assert np.array_equal(got, y)


# the layer's paths: local EC, producer-fused GEMV, semi-fused pairs, k_gemm_r,
# the fused GEMM, 256-token tiles; without an EC the GEMV and the GEMMs
@pytest.mark.parametrize("M,N,K,rank", [(1, 2048, 2048, 16), (4, 4096, 4096, 32), (16, 1024, 4096, 16),
                                        (24, 1024, 4096, 64), (77, 1000, 1408, 24), (300, 512, 2048, 16),
                                        (600, 8192, 512, 16), (3, 520, 1024, 0), (200, 520, 1024, 0)])
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
def test_beside_the_layer(M, N, K, rank, dt):
    from paper_2606_11244_amd import spear as sp
    L, dl = _layer(M, N, K, dt, seed=M, rank=rank)
    s = Slots(M, N, K, 5, 16, dt, seed=9)
    log(f"adapters beside M={M} N={N} K={K} rank={rank} dt={dt}")
    y = _call(dl, s.device(), ec=rank > 0)
    base = O.w4ec_linear(L) if rank else O.w4_linear_layer(L)
    assert_parity(y, base + s.term(_x(dl)), "with adapters")
    # tokens without an adapter get what the plain call writes
    prob = dl.problem()
    plain = torch.empty_like(dl.y)
    (dl.run_ec if rank else dl.run_w4)(prob, sp.allocate_workspace(prob, rank > 0), y=plain)
    torch.cuda.synchronize()
    out = ((s.ids < 0) | (s.ids >= 5)).numpy()
    assert np.array_equal(y[out], plain.double().cpu().numpy()[out])
    none = Slots(M, N, K, 5, 16, dt, ids="none")
    assert np.array_equal(_call(dl, none.device(), ec=rank > 0), plain.double().cpu().numpy())
    zero = Slots(M, N, K, 5, 16, dt)
    zero.ranks = torch.tensor([0, -3, 0, 0, -(2 ** 31)], dtype=torch.int32)
    assert np.array_equal(_call(dl, zero.device(), ec=rank > 0), plain.double().cpu().numpy())


@pytest.mark.parametrize("M,gemm", [(5, 0), (20, 0), (70, 0), (200, 0), (70, 3), (150, 3), (300, 3), (150, 2), (300, 2)])
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
def test_bad_values_stay_with_their_request(M, gemm, dt):
    """Infinities and NaN of one adapter, and of one token, reach no other
    token, and reach their own."""
    with in_the_gemm(gemm) if gemm else contextlib.nullcontext():
        _bad_values(M, dt)


@pytest.mark.parametrize("M,N,K", [(70, 264, 512), (140, 264, 512), (300, 513, 384), (600, 4096, 256)])
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
@pytest.mark.parametrize("roles", [2, 3])
def test_tokens_without_an_adapter_in_the_gemm(M, N, K, dt, roles):
    """They get what the plain call writes there."""
    from paper_2606_11244_amd import spear as sp
    log(f"without an adapter in the GEMM M={M} N={N} K={K} dt={dt}")
    _, dl = _layer(M, N, K, dt, seed=M)
    prob, plain = dl.problem(), torch.empty_like(dl.y)
    with in_the_gemm(roles):
        dl.run_w4(prob, sp.allocate_workspace(prob, False), y=plain)
        torch.cuda.synchronize()
        plain = plain.double().cpu().numpy()
        for ids in ("random", "none"):
            s = Slots(M, N, K, 5, 24, dt, ids=ids, seed=9)
            out = ((s.ids < 0) | (s.ids >= 5)).numpy()
            assert out.any() and np.array_equal(_call(dl, s.device())[out], plain[out])


def _bad_values(M, dt):
    N, K, L, R = 144, 256, 4, 16
    _, dl = _layer(M, N, K, dt, seed=1)
    dl.scales.zero_()
    good = Slots(M, N, K, L, R, dt, ids="turn", seed=6)
    want = _call(dl, good.device()).copy()
    bad = Slots(M, N, K, L, R, dt, ids="turn", seed=6)
    bad.A[1, 3, 7], bad.B[2, 5, 1], bad.scale[3] = INF, NAN, INF
    got = _call(dl, bad.device())
    hit = np.isin(good.ids.numpy(), (1, 2, 3))
    assert np.array_equal(got[~hit], want[~hit])
    assert not np.isfinite(got[hit][good.ids.numpy()[hit] == 1]).all()
    two = good.ids.numpy() == 2
    assert not np.isfinite(got[two][:, 5]).any()
    assert np.array_equal(np.delete(got[two], 5, 1), np.delete(want[two], 5, 1))
    x0 = dl.x.clone()
    dl.x[M // 2, 9] = INF
    got = _call(dl, good.device())
    dl.x.copy_(x0)
    rest = np.arange(M) != M // 2
    # (a layer whose weights are all zero turns that token's product into NaN)
    assert np.array_equal(got[rest], want[rest])


@pytest.mark.parametrize("M,gemm", [(3, 0), (40, 0), (150, 0), (150, 3), (150, 2)])
def test_large_coordinates_in_fp16(M, gemm):
    """Coordinates past the largest fp16 number, and far below the smallest,
    with factors that bring the term back into range."""
    with in_the_gemm(gemm) if gemm else contextlib.nullcontext():
        _large_coordinates(M, gemm)


def _large_coordinates(M, gemm):
    N, K, R = 80, 256, 16
    for up in (2.0 ** 11, 2.0 ** -13):
        _, dl = _layer(M, N, K, S.F16, seed=2)
        dl.scales.zero_()
        s = Slots(M, N, K, 3, R, S.F16, ids="turn", seed=1)
        s.A, s.B = (s.A.float() * up).half(), (s.B.float() / up).half()
        s.scale = s.scale * (64.0 if up > 1 else 1.0 / 64)
        log(f"large coordinates M={M} up={up}")
        y = _call(dl, s.device())
        ref = s.term(_x(dl))
        if up > 1:
            u = O.adapters_term(_x(dl), s.A.double().numpy(), np.eye(R)[None].repeat(3, 0), s.ids, None, s.scale)
            assert np.abs(u).max() > 65504
        lim = s.bound(_x(dl), ref, ref)
        if gemm:  # unscaled small coordinates: each off by at most 2^-25
            lim = lim + 2.0 ** -25 * np.abs(s.B.double().numpy()).sum(2)[s.ids.numpy()]
        assert np.all(np.abs(y - ref) <= lim), (np.abs(y - ref) / lim).max()


GROUPS = [
    # (M, N, K, EC rank, adapters' (L, R) or None) of each member
    [(1, 256, 512, 16, (3, 8)), (1, 128, 512, 16, (3, 8)), (1, 128, 512, 16, None)],
    [(16, 1024, 1024, 0, (20, 16)), (16, 256, 1024, 0, (20, 16)), (16, 256, 1024, 0, (4, 64))],
    [(24, 512, 4096, 64, (9, 32)), (24, 512, 4096, 64, (9, 32))],
    [(48, 1024, 2048, 0, (6, 16)), (48, 1024, 2048, 32, (6, 24)), (3, 136, 256, 0, (2, 5))],
    [(2048, 8192, 128, 0, (3, 16)), (2048, 8200, 128, 0, (4, 40)), (70, 64, 128, 0, (3, 8))],
    [(48, 520, 1024, 32, (6, 16)), (48, 264, 1024, 32, (48, 24)), (48, 136, 1024, 24, None), (40, 520, 1024, 32, (2, 8))],
    [(1, 4096, 4096, 64, (2, 16)), (1, 1024, 4096, 64, (2, 16)), (1, 1024, 4096, 64, None)],
    [(12, 1024, 4096, 64, (5, 16)), (12, 4096, 4096, 64, (5, 40))],
    [(200, 520, 512, 0, (3, 16)), (0, 64, 256, 0, (2, 4)), (200, 264, 512, 16, None), (70, 64, 256, 0, (9, 12))],
]


@pytest.mark.parametrize("spec", GROUPS)
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
def test_group_equals_single_calls(spec, dt):
    from paper_2606_11244_amd import spear as sp
    members, want = [], []
    for i, (M, N, K, rank, lr) in enumerate(spec):
        L, dl = _layer(max(M, 1), N, K, dt, seed=i, rank=rank)
        prob = dl.problem()
        prob.M = M
        m = dl.member(prob, with_ec=rank > 0)
        m["y"] = torch.full((M + 1, N), 7.0, dtype=DT[dt], device="cuda")
        m["adapters"] = Slots(max(M, 1), N, K, *lr, dt, seed=i, mixed=True).device() if lr else None
        members.append(m)
        y = torch.full_like(m["y"], 7.0)
        if M:
            ad = m["adapters"] or sp.adapters(*(torch.empty(0, *d, dtype=DT[dt], device="cuda") for d in ((1, K), (N, 1))),
                                              torch.zeros(M, dtype=torch.int32, device="cuda"))
            ws = torch.zeros(sp.adapters_workspace([dict(m, adapters=ad)]), dtype=torch.uint8, device="cuda")
            sp.w4ec_linear_adapters(prob, m["x"], m["qweight"], m["scales"], m["zeros"], ad, y,
                                    ec_args=m["ec_args"], workspace=ws)
        want.append(y)
    log(f"adapters group {spec} dt={dt}")
    ws = torch.zeros(sp.adapters_workspace(members), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        sp.w4ec_linear_adapters_group(members, ws)
        torch.cuda.synchronize()
        for m, y in zip(members, want):
            assert torch.equal(m["y"], y)


@pytest.mark.parametrize("M,R", [(4, 16), (16, 64), (90, 16)])
def test_graph_follows_the_batch(M, R):
    """A captured group replays with other inputs, adapters and ids, between
    eager calls on the same workspace."""
    from paper_2606_11244_amd import spear as sp
    N, K, dt = 264, 1024, S.F16
    dls = [_layer(M, N, K, dt, seed=i, rank=16)[1] for i in range(2)]
    slots = [[Slots(M, N, K, 6, R, dt, seed=10 * j + i, ids="turn" if j else "random") for i in range(2)]
             for j in range(4)]
    ads = [slots[0][i].device() for i in range(2)]
    members = [dict(d.member(d.problem()), adapters=a) for d, a in zip(dls, ads)]
    ws = torch.zeros(sp.adapters_workspace(members), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sp.w4ec_linear_adapters_group(members, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.w4ec_linear_adapters_group(members, ws)
    xs = [torch.randn(M, K, device="cuda").half() for _ in range(4)]
    for j in (1, 2, 3, 0, 2):
        log(f"adapters replay {j} M={M} R={R}")
        for i in range(2):
            dls[i].x.copy_(xs[j])
            A, B, ids, _, scale = ads[i]._keep
            A.copy_(slots[j][i].A), B.copy_(slots[j][i].B), ids.copy_(slots[j][i].ids), scale.copy_(slots[j][i].scale)
        graph.replay()
        torch.cuda.synchronize()
        got = [m["y"].clone() for m in members]
        for m, y in zip(members, got):
            eager = torch.empty_like(y)
            sp.w4ec_linear_adapters(m["prob"], m["x"], m["qweight"], m["scales"], m["zeros"], m["adapters"],
                                    eager, ec_args=m["ec_args"], workspace=ws)
            torch.cuda.synchronize()
            assert torch.equal(eager, y)


def test_another_stream_and_far_slots():
    """A call on a stream of its own; slots whose last lies past 2^32 bytes."""
    from paper_2606_11244_amd import spear as sp
    M, N, K, R, dt = 20, 136, 256, 16, S.BF16
    _, dl = _layer(M, N, K, dt, seed=3)
    dl.scales.zero_()
    s = Slots(M, N, K, 3, R, dt, ids="turn", seed=4)
    stride = (1 << 30) + 64  # elements: slot 2 at 4 GiB
    need = 2 * stride + N * K
    far = torch.empty(need, dtype=DT[dt], device="cuda")
    A, B = (far.as_strided(t.shape, (stride, t.shape[2], 1), o) for t, o in ((s.A, 0), (s.B, R * K)))
    A.copy_(s.A), B.copy_(s.B)
    ad = sp.adapters(A, B, s.ids.cuda(), scale=s.scale.cuda())
    ref = s.term(_x(dl))
    m = dict(dl.member(dl.problem(), with_ec=False), adapters=ad)
    ws = torch.zeros(sp.adapters_workspace([m]), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    sp.w4ec_linear_adapters(m["prob"], dl.x, dl.qweight, dl.scales, dl.zeros, ad, dl.y, workspace=ws, stream=st)
    st.synchronize()
    assert np.all(np.abs(dl.y.double().cpu().numpy() - ref) <= s.bound(_x(dl), ref, ref))


@pytest.mark.parametrize("M,N,K,L,R", [(1, 520, 1152, 3, 16), (16, 256, 1024, 16, 16), (27, 1000, 512, 5, 40), (32, 130, 256, 40, 8)])
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
def test_one_rounding_at_decode(M, N, K, L, R, dt):
    """The layer, the term and the residual meet before y is rounded. Small integers
    and powers of two: every sum is exact in fp32 (up to 2^22 in steps of one before
    the powers), u in two parts too, and y is the exact sum rounded once; from 17
    tokens on, where the layer is a GEMM, the term with the residual is rounded too."""
    from paper_2606_11244_amd import spear as sp
    lay, dl = _layer(M, N, K, dt, seed=M)
    g = torch.Generator().manual_seed(K)
    dl.x.copy_(torch.randint(-2, 3, (M, K), generator=g))
    bits = np.full_like(lay.scales, np.float16(2.0 ** -6).view(np.uint16))
    dl.scales.copy_(torch.from_numpy(bits.view(np.int16)).view(dl.scales.dtype))
    s = Slots(M, N, K, L, R, dt, ids="turn", seed=5)
    s.A.copy_(torch.randint(-1, 2, s.A.shape, generator=g))
    s.B.copy_(torch.randint(-3, 4, s.B.shape, generator=g) * 2.0 ** -7)
    s.scale = 2.0 ** torch.randint(-1, 2, (L,), generator=g).float()
    res = (torch.randint(-99, 100, (M, N), generator=g) * 2.0 ** -6).to(DT[dt])
    log(f"one rounding M={M} N={N} K={K} L={L} R={R} dt={dt}")
    y = _call(dl, s.device(), residual=res.cuda())
    W = O.dequant(lay.qweight, bits, lay.zeros, lay.group_size)
    assert np.abs(W).max() >= 2.0 ** -4

    def rounded(v):
        assert np.array_equal(v, np.float32(v))
        return torch.from_numpy(v).float().to(DT[dt]).double().numpy()
    rest = s.term(_x(dl)) + res.double().numpy()
    gemv = sp.dispatch_plan(dl.problem(), with_ec=False).path == sp.PATH_FUSED_GEMV
    assert gemv or M > 16
    assert np.array_equal(y, rounded(O.w4_linear(_x(dl), W) + (rest if gemv else rounded(rest))))


MIXED = [
    # (M, N, K, EC rank, weight bits, INT8 factors, dtype, adapters (L, R)) of each member
    [(4, 256, 512, 16, 4, False, S.F16, (3, 8)), (4, 256, 512, 16, 4, False, S.BF16, (3, 8)),
     (4, 128, 512, 0, 3, False, S.F16, (2, 16)), (20, 64, 256, 0, 4, False, S.F16, None)],
    [(8, 512, 1024, 16, 4, True, S.F16, (8, 16)), (8, 512, 1024, 16, 4, True, S.F16, None),
     (8, 512, 1024, 0, 4, False, S.F16, (8, 24)), (40, 512, 1024, 0, 3, False, S.BF16, (8, 16))],
    [(1, 4096, 1024, 0, 4, False, S.F16, (2, 8)), (30, 128, 1024, 0, 4, False, S.F16, (30, 8)),
     (64, 128, 1024, 32, 4, False, S.F16, (5, 8)), (65, 128, 1024, 0, 4, False, S.F16, (5, 8))],
    [(48, 520, 1024, 32, 4, True, S.F16, (6, 16)), (100, 264, 1024, 32, 4, True, S.F16, (100, 8)),
     (128, 264, 1024, 32, 3, False, S.F16, (3, 40)), (129, 264, 1024, 32, 4, False, S.BF16, (3, 40))],
]


def _mixed(spec, seed=0):
    from paper_2606_11244_amd import spear as sp
    members = []
    for i, (M, N, K, rank, bits, i8, dt, lr) in enumerate(spec):
        kw = dict(weight_bits=bits) if bits != 4 else {}
        if i8:
            kw["ab_int8"] = True
        _, dl = _layer(M, N, K, dt, seed=seed + i, rank=rank, **kw)
        m = dl.member(dl.problem(), with_ec=rank > 0)
        m["y"] = torch.full((M, N), 7.0, dtype=DT[dt], device="cuda")
        m["adapters"] = Slots(M, N, K, *lr, dt, seed=i).device() if lr else None
        members.append(m)
    return sp, members


def _singly(sp, m, ws=None):
    M, K, N = m["prob"].M, m["prob"].K, m["prob"].N
    t = m["y"].dtype
    ad = m["adapters"] or sp.adapters(torch.empty(0, 1, K, dtype=t, device="cuda"), torch.empty(0, N, 1, dtype=t, device="cuda"),
                                      torch.zeros(M, dtype=torch.int32, device="cuda"))
    if ws is None:
        ws = torch.zeros(sp.adapters_workspace([dict(m, adapters=ad)]), dtype=torch.uint8, device="cuda")
    y = torch.empty_like(m["y"])
    sp.w4ec_linear_adapters(m["prob"], m["x"], m["qweight"], m["scales"], m["zeros"], ad, y, ec_args=m["ec_args"], workspace=ws)
    torch.cuda.synchronize()
    return y


@pytest.mark.parametrize("spec", MIXED)
def test_groups_of_unlike_members(spec):
    """Code widths, activation dtypes, INT8 factors, members that share no launch."""
    sp, members = _mixed(spec)
    want = [_singly(sp, m) for m in members]
    ws = torch.zeros(sp.adapters_workspace(members), dtype=torch.uint8, device="cuda")
    for order in ([0, 1, 2, 3], [3, 1, 0, 2], [2, 3, 1, 0]):
        log(f"mixed group {spec} order {order}")
        for m in members:
            m["y"].fill_(7.0)
        group = [members[i] for i in order]
        assert sp.adapters_workspace(group) == ws.numel()
        sp.w4ec_linear_adapters_group(group, ws)
        torch.cuda.synchronize()
        for m, y in zip(members, want):
            assert torch.equal(m["y"], y)


@pytest.mark.parametrize("stages,shape", [(4, None), (2, (2, 2, 4)), (None, (1, 3, 8))])
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
def test_other_launch_shapes_of_the_layer(stages, shape, dt):
    """K-slices, row tiles and pipelines of the decode GEMV other than the planner's."""
    from paper_2606_11244_amd import spear as sp
    M, N, K = 9, 520, 2048
    lay, dl = _layer(M, N, K, dt, seed=4)
    s = Slots(M, N, K, 4, 16, dt, seed=4)
    log(f"adapters stages {stages} shape {shape} dt={dt}")
    try:
        if stages:
            sp.set_gemv_stages(stages)
        if shape:
            sp.set_gemv_shape(*shape)
        y = _call(dl, s.device())
    finally:
        sp.set_gemv_stages(0)
        sp.set_gemv_shape(0, 0, 0)
    x = _x(dl)
    assert_parity(y, O.w4_linear(x, O.dequant(lay.qweight, lay.scales, lay.zeros, lay.group_size)) + s.term(x), "launch shapes")


def test_two_graphs_share_a_workspace():
    """Captured calls of different shapes on one workspace, replayed in turn."""
    from paper_2606_11244_amd import spear as sp
    sets = [_mixed(spec, seed=20 * k)[1] for k, spec in enumerate(MIXED)]
    want = [[_singly(sp, m) for m in ms] for ms in sets]
    ws = torch.zeros(max(sp.adapters_workspace(ms) for ms in sets), dtype=torch.uint8, device="cuda")
    graphs = []
    for ms in sets:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            sp.w4ec_linear_adapters_group(ms, ws)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sp.w4ec_linear_adapters_group(ms, ws)
        graphs.append(g)
    for k in (0, 1, 2, 1, 0, 0, 2, 1):
        log(f"two graphs: {k}")
        for m in sets[k]:
            m["y"].fill_(7.0)
        graphs[k].replay()
        torch.cuda.synchronize()
        for m, y in zip(sets[k], want[k]):
            assert torch.equal(m["y"], y)


def test_two_calls_at_once():
    """Two streams, the same weights and adapters, a workspace each."""
    sp, members = _mixed(MIXED[2])
    want = [_singly(sp, m) for m in members]
    streams = [torch.cuda.Stream() for _ in range(2)]
    other = [dict(m, y=torch.empty_like(m["y"])) for m in members]
    ws = [torch.zeros(sp.adapters_workspace(members), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    log("two calls at once")
    for _ in range(5):
        for ms, w, st in zip((members, other), ws, streams):
            sp.w4ec_linear_adapters_group(ms, w, stream=st)
    torch.cuda.synchronize()
    for ms in (members, other):
        for m, y in zip(ms, want):
            assert torch.equal(m["y"], y)
