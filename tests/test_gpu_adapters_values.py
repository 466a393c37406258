"""GPU tests of what a token's result may depend on, and of how far it may be off,
where adapters meet the layer's kernels: its companions in the batch, the number
of roundings, values that are not finite."""
from __future__ import annotations

import contextlib

import numpy as np
import pytest
import torch

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
