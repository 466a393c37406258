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

from gpu_util import log
from test_gpu_adapters import DT, Slots, _call, _gpu, _layer, in_the_gemm  # noqa: F401 (a fixture)

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
