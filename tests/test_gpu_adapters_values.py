"""GPU tests of what a token's result may depend on, and of how far it may be off,
where adapters meet the layer's kernels: its companions in the batch, the number
of roundings, values that are not finite."""
from __future__ import annotations

import contextlib

import numpy as np
import pytest
import torch

from oracle import spear_oracle as O
from paper_2606_11244_amd import synth as S

from gpu_util import assert_parity, log
from test_gpu_adapters import DT, HALF, Slots, _call, _gpu, _layer, _x, in_the_gemm  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


# (M, N, K, EC rank, the GEMM's roles): the coordinates beside a GEMV and a local EC,
# by themselves, beside an EC pre-kernel, by slots and by tiles of 64 tokens, and the
# term in the GEMM; K in several iterations a wave and slice
COMPANY = [(3, 264, 8192, 0, 0), (16, 264, 4096, 0, 0), (8, 520, 4096, 16, 0), (9, 512, 8192, 48, 0),
           (24, 520, 4096, 64, 0), (33, 264, 4096, 0, 0), (64, 264, 4096, 32, 0), (100, 136, 4096, 0, 0),
           (200, 136, 4096, 0, 0), (300, 264, 4096, 0, 3)]


@pytest.mark.parametrize("M,N,K,rank,roles", COMPANY)
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
def test_a_token_does_not_see_its_companions(M, N, K, rank, roles, dt):
    """Bit for bit the same, whichever adapters the other tokens have, and, of the
    adapters' term, whichever row of the batch the token lies in."""
    _, dl = _layer(M, N, K, dt, seed=M, rank=rank)
    L, R, a = 6, 24, 4
    s = Slots(M, N, K, L, R, dt, seed=3)
    token = M - 1
    with in_the_gemm(roles) if roles else contextlib.nullcontext():
        want = None
        for what in ("turn", "all", "none", "half", "last"):
            ids = torch.arange(M) % L
            if what == "all":
                ids[:] = a
            elif what == "none":
                ids[:] = -1
            elif what == "half":
                ids[::2] = a
            elif what == "last":
                ids[M // 2:] = a
            ids[token] = a
            s.ids = ids.to(torch.int32)
            log(f"companions {what} M={M} N={N} K={K} rank={rank} roles={roles} dt={dt}")
            y = _call(dl, s.device(), ec=rank > 0)[token].copy()
            want = y if want is None else want
            assert np.array_equal(y, want), what
        if rank:
            return
        dl.scales.zero_()
        s.ids = (torch.arange(M) * 5 % (L + 1) - 1).to(torch.int32)
        x, ids = dl.x.clone(), s.ids.clone()
        y = _call(dl, s.device()).copy()
        for seed in (1, 2):
            perm = torch.randperm(M, generator=torch.Generator().manual_seed(seed))
            dl.x.copy_(x[perm.cuda()])
            s.ids = ids[perm].contiguous()
            log(f"order {seed} M={M} N={N} K={K} roles={roles} dt={dt}")
            assert np.array_equal(_call(dl, s.device()), y[perm.numpy()])


# (M, N, K, EC rank, path): the local EC, the producer-fused GEMV and the semi-fused one
DECODE_EC = [(1, 130, 256, 8, "LOCAL"), (5, 520, 1024, 16, "LOCAL"), (1, 520, 1152, 64, "GEMV"), (8, 264, 4608, 48, "GEMV"),
             (24, 264, 4608, 64, "GEMV"), (4, 520, 1024, 32, "2K"), (16, 264, 2048, 64, "2K")]


def _path(dl):
    from paper_2606_11244_amd import spear as sp
    path = sp.dispatch_plan(dl.problem(), with_ec=True).path
    return {sp.PATH_FUSED_LOCAL: "LOCAL", sp.PATH_FUSED_GEMV: "GEMV", sp.PATH_UNFUSED_2K: "2K"}.get(path)


@pytest.mark.parametrize("M,N,K,rank,path", DECODE_EC)
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
def test_one_rounding_at_decode_with_an_ec(M, N, K, rank, path, dt):
    """Layer, EC, term and residual meet before y is rounded. Small integers and
    powers of two: the product's sums are at most 4608 * 2 * (1024 + 15) < 2^24 in
    steps of one, everything else lies in steps of 2^-8 below 2^15, so that every sum
    is exact in fp32 and y is the exact sum rounded once."""
    lay, dl = _layer(M, N, K, dt, seed=M, rank=rank, gate_kind=S.GATE_ONE)
    assert _path(dl) == path
    g = torch.Generator().manual_seed(K + rank)
    dl.x.copy_(torch.randint(-2, 3, (M, K), generator=g))
    bits = np.full_like(lay.scales, np.float16(2.0 ** -6).view(np.uint16))
    dl.scales.copy_(torch.from_numpy(bits.view(np.int16)).view(dl.scales.dtype))
    lay.alpha = 1.0
    dl.A.copy_(torch.randint(-1, 2, dl.A.shape, generator=g))
    dl.B.copy_(torch.randint(-3, 4, dl.B.shape, generator=g) * 2.0 ** -7)
    s = Slots(M, N, K, 4, 24, dt, ids="turn", seed=5)
    s.A.copy_(torch.randint(-1, 2, s.A.shape, generator=g))
    s.B.copy_(torch.randint(-3, 4, s.B.shape, generator=g) * 2.0 ** -7)
    s.scale = 2.0 ** torch.randint(-1, 2, (4,), generator=g).float()
    res = (torch.randint(-99, 100, (M, N), generator=g) * 2.0 ** -6).to(DT[dt])
    log(f"one rounding with an EC M={M} N={N} K={K} rank={rank} dt={dt}")
    y = _call(dl, s.device(), ec=True, residual=res.cuda())
    x = dl.x.double().cpu().numpy()
    W = O.dequant(lay.qweight, bits, lay.zeros, lay.group_size)
    want = O.w4_linear(x, W) + (x @ dl.A.double().cpu().numpy().T) @ dl.B.double().cpu().numpy().T
    want = want + s.term(x) + res.double().numpy()
    assert np.array_equal(want, np.float32(want)) and np.abs(want).max() < 2.0 ** 15
    assert np.array_equal(y, torch.from_numpy(want).float().to(DT[dt]).double().numpy())
    assert np.array_equal(_call(dl, s.device(), ec=True, residual=res.cuda()), y)  # (the workspace's counters go on)


@pytest.mark.parametrize("M,N,K,rank,path", [(1, 264, 1152, 48, "GEMV"), (9, 264, 4608, 40, "GEMV"), (6, 264, 1024, 32, "2K"),
                                             (20, 130, 4608, 64, "GEMV")])
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
@pytest.mark.parametrize("bits,int8,gate", [(3, False, S.GATE_SIGMOID_LINEAR), (4, True, S.GATE_SIGMOID_LINEAR), (3, True, S.GATE_TANH_MLP)])
def test_an_ec_wave_of_other_kinds(M, N, K, rank, path, dt, bits, int8, gate):
    """Three-bit codes, INT8 factors and the tanh-MLP gate beside adapters at decode."""
    L, dl = _layer(M, N, K, dt, seed=M, rank=rank, weight_bits=bits, ab_int8=int8, gate_kind=gate)
    assert _path(dl) == path
    s = Slots(M, N, K, 5, 16, dt, seed=9, mixed=True)
    log(f"EC wave M={M} N={N} K={K} rank={rank} bits={bits} int8={int8} gate={gate} dt={dt}")
    assert_parity(_call(dl, s.device(), ec=True), O.w4ec_linear(L) + s.term(_x(dl)), "an EC wave")


@pytest.mark.parametrize("M,K,rank,path", [(1, 1152, 64, "GEMV"), (8, 4608, 48, "GEMV"), (4, 1024, 32, "2K")])
def test_replays_with_an_ec_wave(M, K, rank, path):
    """A captured call and group, replayed with other inputs between eager calls of
    the same and of another layer on the same workspace."""
    from paper_2606_11244_amd import spear as sp
    N, dt = 264, S.F16
    dls = [_layer(M, N, K, dt, seed=i, rank=rank)[1] for i in range(3)]
    assert _path(dls[0]) == path
    members = [dict(d.member(d.problem()), adapters=Slots(M, N, K, 4, 24, dt, seed=i).device()) for i, d in enumerate(dls)]
    ws = torch.zeros(sp.adapters_workspace(members), dtype=torch.uint8, device="cuda")

    def single(m, y):
        sp.w4ec_linear_adapters(m["prob"], m["x"], m["qweight"], m["scales"], m["zeros"], m["adapters"], y,
                                ec_args=m["ec_args"], workspace=ws)

    def run():
        single(members[0], members[0]["y"])
        sp.w4ec_linear_adapters_group(members[1:], ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for j in range(4):
        log(f"replay {j} with an EC wave M={M} K={K} rank={rank}")
        for d in dls:
            d.x.copy_(torch.randn(M, K, generator=torch.Generator().manual_seed(j)))
        graph.replay()
        torch.cuda.synchronize()
        for m in members:
            eager = torch.empty_like(m["y"])
            single(m, eager)
            torch.cuda.synchronize()
            assert torch.equal(eager, m["y"])
            m["y"].zero_()


@pytest.mark.parametrize("M,N,K,rank,path", DECODE_EC + [(3, 264, 1152, 0, None)])
def test_decode_sums_pass_the_range_of_fp16(M, N, K, rank, path):
    """The residual and the term together are beyond fp16's largest number, the
    layer brings them back: 60000 + 100 * 200 - 8 * 30000 / (8 K) * K."""
    lay, dl = _layer(M, N, K, S.F16, seed=M, rank=rank, gate_kind=S.GATE_ONE)
    assert not rank or _path(dl) == path
    dl.x.fill_(1.0)
    dl.qweight.zero_()
    dl.zeros.fill_(8)
    step = torch.tensor(30000.0 / (8 * K)).half()
    dl.scales.copy_(torch.full(dl.scales.shape, step.item(), dtype=torch.float16).view(dl.scales.dtype))
    if rank:
        dl.B.zero_()
    s = Slots(M, N, K, 2, 8, S.F16, ids="turn", scale=False)
    s.A.zero_(), s.B.zero_()
    s.A[:, 1, :100], s.B[:, :, 1] = 1.0, 200.0
    res = torch.full((M, N), 60000.0, dtype=torch.float16)
    log(f"past fp16 M={M} N={N} K={K} rank={rank}")
    y = _call(dl, s.device(), ec=rank > 0, residual=res.cuda())
    want = 80000.0 - 8.0 * K * step.item()
    # half a step of fp16 there, and a rounding of 2^-24 a step of the sums over K
    assert np.all(np.abs(y - want) <= 16.0 + K * 2.0 ** -24 * 110000.0)


def _kind(v):
    return np.where(np.isnan(v), 2.0, np.where(np.isinf(v), np.sign(v), 0.0))


@pytest.mark.parametrize("M,N,roles", [(150, 144, 2), (150, 144, 3), (300, 520, 2), (300, 520, 3)])
@pytest.mark.parametrize("dt", [S.F16, S.BF16])
@pytest.mark.parametrize("residual", [False, True])
def test_what_is_not_finite_in_b_keeps_its_kind_in_the_gemm(M, N, roles, dt, residual):
    """NaN, infinities of both signs and of both on one row, where the GEMM forms the
    term: as the formula gives them, on their own rows and tokens only."""
    K, L, R = 256, 4, 40
    _, dl = _layer(M, N, K, dt, seed=1)
    dl.scales.zero_()
    s = Slots(M, N, K, L, R, dt, ids="turn", seed=6)
    res = torch.randn(M, N, generator=torch.Generator().manual_seed(3)).to(DT[dt]) if residual else None
    kw = dict(residual=res.cuda()) if residual else {}
    with in_the_gemm(roles):
        want = _call(dl, s.device(), **kw).copy()
        s.B[1, 3, 35], s.B[1, 130, 2], s.B[2, 7, 5] = np.nan, np.inf, -np.inf
        s.B[2, N - 1, 1], s.B[2, N - 1, 39], s.B[3, 0, 0], s.B[3, 0, 1] = np.inf, -np.inf, np.inf, np.nan
        log(f"not finite M={M} N={N} roles={roles} dt={dt} residual={residual}")
        inplace = kw["residual"] if residual else None
        got = _call(dl, s.device(), y=inplace, **kw) if residual else _call(dl, s.device())
    A, B, x = s.A.double().numpy(), s.B.double().numpy(), _x(dl)
    with np.errstate(invalid="ignore"):
        ref = np.stack([(float(s.scale[a]) * (x[m] @ A[a].T) * B[a]).sum(1) for m, a in enumerate(s.ids.tolist())])
    assert (_kind(ref) != 0).sum() >= M and {2.0, 1.0, -1.0} <= set(_kind(ref).ravel())
    assert np.array_equal(_kind(got), _kind(ref))
    fine = np.isfinite(ref)
    assert np.array_equal(got[fine], want[fine])


@pytest.mark.parametrize("M,N,roles", [(150, 144, 2), (150, 144, 3), (300, 520, 3)])
def test_entries_past_the_range_of_fp16_in_the_gemm(M, N, roles):
    """A coordinate of 2^20 is divided by 2^6 there and the slot's B multiplied by it,
    which entries of 2000 do not bear: y is finite all the same, either sign. Powers of
    two and small integers: but for two roundings of y, and one for the pair of an
    entry that was kept out, everything is exact."""
    K, R = 256, 8
    _, dl = _layer(M, N, K, S.F16, seed=1)
    dl.scales.zero_()
    dl.x.fill_(1.0)
    s = Slots(M, N, K, 2, R, S.F16, ids="turn", scale=False)
    s.A.zero_()
    s.A[:, 0], s.A[:, 1, :2], s.A[:, 2, 0] = 4096.0, 1.0, -1.0  # coordinates 2^20, 2, -1
    s.B.zero_()
    s.B[:, :, 0] = 2.0 ** -8 * (1 + torch.arange(N) % 3)  # the term 4096, 8192, 12288
    s.B[0, 5::16, 1] = 2000.0                              # + 4000
    s.B[1, 6::16, 2] = 1504.0                              # - 1504
    s.B[1, 7::16, 2] = -2000.0                             # + 2000
    log(f"past fp16 in the GEMM M={M} N={N} roles={roles}")
    with in_the_gemm(roles):
        y = _call(dl, s.device())
    ref = s.term(_x(dl))
    assert np.abs(ref).max() < 2.0 ** 15 and (ref != ref[0]).any()
    # half a step of fp16 for each rounding: of the partial sum and of y
    assert np.all(np.abs(y - ref) <= HALF[S.F16] * (np.abs(ref) + 4000.0 + np.abs(ref)))
    alone = np.ones(N, bool)
    alone[5::16] = alone[6::16] = alone[7::16] = False
    assert np.array_equal(y[:, alone], ref[:, alone])
