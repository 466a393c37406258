"""GPU parity of the norms around a block against the float64 oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import spear_oracle as O
from paper_2606_11244_amd import synth as S

from gpu_util import log

pytestmark = pytest.mark.gpu

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _rows(t, pad):
    """t on the GPU with `pad` elements of NaN between its rows."""
    if not pad:
        return t.cuda()
    buf = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    buf[:, :t.shape[1]] = t.cuda()
    return buf[:, :t.shape[1]]


def _case(M, N, dt, *, f32=False, post=True, pre=True, gates="one", kind="mul", stream=True, rho=1.0, beta=1.0,
          off=0.0, eps=1e-5, pad=0, seed=0, mag=3.0):
    g = torch.Generator().manual_seed(seed + 131 * M + N)

    def rnd(*s):
        return torch.randn(*s, generator=g)
    c = dict(M=M, N=N, dt=dt, f32=f32, kind=kind, rho=rho, beta=beta, off=off, eps=eps, pad=pad)
    c["y"] = (rnd(M, N) * mag).to(dt)
    c["h"] = rnd(M, N).to(torch.float32 if f32 else dt) if stream else None
    c["post_w"] = (1 - off + 0.2 * rnd(N)).to(dt) if post else None
    c["pre_w"] = (1 - off + 0.2 * rnd(N)).to(dt) if pre else None
    n = {"none": 0, "one": 1, "row": M, "ids": max(1, M // 2)}[gates]
    c["gate"] = rnd(n, N).to(dt) if n else None
    c["gate_ids"] = torch.randint(-1, n + 1, (M,), generator=g, dtype=torch.int32) if gates == "ids" else None
    return c


def _run(c, h_out=None, h=None):
    from paper_2606_11244_amd import spear as sp
    M, N, pad = c["M"], c["N"], c["pad"]
    sdt = torch.float32 if c["f32"] else c["dt"]

    def cu(t):
        return None if t is None else t.cuda()
    if h_out is None:
        h_out = _rows(torch.full((M + 1, N), 5.0, dtype=sdt), pad)
    x = _rows(torch.full((M + 1, N), 5.0, dtype=c["dt"]), pad)
    h = h if h is not None else None if c["h"] is None else _rows(c["h"], pad)
    sp.block_norm(_rows(c["y"], pad), h, h_out[:M], x[:M] if c["pre_w"] is not None else None,
                  post_w=cu(c["post_w"]), pre_w=cu(c["pre_w"]),
                  gate=None if c["gate"] is None else _rows(c["gate"], pad), gate_ids=cu(c["gate_ids"]),
                  gate_kind=c["kind"], stream_scale=c["rho"], branch_scale=c["beta"], w_offset=c["off"], eps=c["eps"])
    torch.cuda.synchronize()
    # rows behind the last, and what lies between strided rows, as they were
    for t in (h_out, x):
        if t.shape[0] > M:
            assert torch.all(t[M:] == 5.0)
        if pad and M:
            assert torch.isnan(t.as_strided((M, pad), (N + pad, 1), t.storage_offset() + N)).all()
    assert c["pre_w"] is not None or torch.all(x == 5.0)
    return h_out[:M].double().cpu().numpy(), x[:M].double().cpu().numpy()


def _np(t):
    return None if t is None else t.double().numpy()


def _check(c, h_out, x):
    """h': half a step of its type, and fp32 arithmetic: a sum of N squares (N
    roundings), some ten further operations and the exponential functions (four
    steps), each relative to the magnitudes added. x: of the stored h'."""
    N = c["N"]
    args = (_np(c["y"]), _np(c["h"]), _np(c["post_w"]), _np(c["gate"]), c["gate_ids"], c["kind"])
    ref = O.block_stream(*args, c["rho"], c["beta"], c["eps"], c["off"])
    o = O.block_stream(args[0], None, *args[2:], 1.0, abs(c["beta"]), c["eps"], c["off"])
    mag = np.abs(o) + (0 if c["h"] is None else np.abs(c["rho"] * args[1]))
    f = (N / 2 + 16) * 2.0 ** -24
    tiny = 2.0 ** -24 if not c["f32"] and c["dt"] == torch.float16 else 1e-37
    lim = f * mag + HALF[torch.float32 if c["f32"] else c["dt"]] * 1.001 * np.abs(ref) + tiny
    err = np.abs(h_out - ref)
    assert np.all(err <= lim), ("h", err.max(), (err / lim).max())
    if c["pre_w"] is None:
        return
    want = O.rms_norm(h_out, _np(c["pre_w"]), c["eps"], c["off"])
    lim = (f + HALF[c["dt"]] * 1.001) * np.abs(want) + (2.0 ** -24 if c["dt"] == torch.float16 else 1e-37)
    err = np.abs(x - want)
    assert np.all(err <= lim), ("x", err.max(), (err / lim).max())


SIZES = [(1, 1), (1, 8), (3, 7), (2, 64), (5, 65), (70, 128), (9, 500), (130, 512), (4, 520), (33, 1024), (3, 1030),
         (7, 2048), (2, 2056), (17, 4096), (5, 4104), (24, 8192), (3, 8200), (2, 16384), (2, 16400), (1, 32768),
         (2, 32776), (3, 40001), (1000, 16), (4097, 64)]


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("f32", [False, True])
def test_sizes(M, N, dt, f32):
    log(f"block norm M={M} N={N} dt={dt} f32={f32}")
    c = _case(M, N, dt, f32=f32, gates="row" if M % 2 else "one", kind=("mul", "tanh", "sigmoid")[N % 3], rho=0.75, beta=1.5)
    _check(c, *_run(c))


FORMS = [
    dict(post=False, gates="none"), dict(pre=False), dict(post=False, pre=False, gates="none", rho=0.5),
    dict(stream=False), dict(stream=False, post=False, gates="none", pre=False, beta=-2.0),
    dict(gates="ids", kind="tanh"), dict(gates="ids", kind="sigmoid", pad=8), dict(gates="row", kind="tanh", pad=8),
    dict(off=1.0), dict(off=1.0, pre=False, gates="ids"), dict(pad=3), dict(pad=1, gates="row", kind="sigmoid"),
    dict(rho=0.0), dict(beta=0.0), dict(eps=0.0), dict(eps=1.0, rho=-1.25),
]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("M,N", [(6, 2048), (6, 200), (6, 203), (5, 5120), (300, 96)])
@pytest.mark.parametrize("dt,f32", [(torch.float16, False), (torch.bfloat16, False), (torch.bfloat16, True)])
def test_forms(form, M, N, dt, f32):
    log(f"block norm {form} M={M} N={N} dt={dt} f32={f32}")
    c = _case(M, N, dt, f32=f32, seed=3, **form)
    _check(c, *_run(c))


@pytest.mark.parametrize("M,N", [(40, 2048), (40, 203), (200, 96), (3, 40000)])
@pytest.mark.parametrize("f32", [False, True])
def test_in_place(M, N, f32):
    """h_out is h itself."""
    c = _case(M, N, torch.float16, f32=f32, gates="one")
    want = _run(c)
    h = c["h"].cuda()
    got = _run(c, h_out=h, h=h)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


@pytest.mark.parametrize("M,N", [(8, 2048), (8, 203), (64, 96), (5, 20000)])
def test_bad_values_stay_in_their_row(M, N):
    c = _case(M, N, torch.bfloat16, gates="row", kind="sigmoid", seed=1)
    want = _run(c)
    c["y"][1, N // 2], c["h"][2, 0], c["gate"][3, N - 1] = float("inf"), float("nan"), float("nan")
    c["gate"][4] = float("inf")   # a gate fully open, and fully shut
    c["gate"][0] = -float("inf")
    got = _run(c)
    for a, b in zip(got, want):
        assert np.array_equal(a[5:], b[5:])
        assert np.isfinite(a[[0, 4]]).all()
    assert np.isnan(got[0][1]).any() and np.isnan(got[0][2, 0]) and np.isnan(got[0][3, N - 1])
    assert np.isnan(got[1][2]).all() and np.isnan(got[1][3]).all()
    assert np.array_equal(got[0][0], c["h"][0].double().numpy())


def test_row_of_zeros():
    c = _case(4, 1024, torch.float16, gates="none")
    c["y"][1] = 0.0
    c["y"][2], c["h"][2] = 0.0, 0.0
    h, x = _run(c)
    assert np.array_equal(h[1], c["h"][1].double().numpy()) and not h[2].any() and not x[2].any()
    _check(c, h, x)


def test_replays_follow_the_batch():
    from paper_2606_11244_amd import spear as sp
    M, N = 9, 2048
    cs = [_case(M, N, torch.float16, gates="ids", kind="tanh", seed=s) for s in range(3)]
    b = {k: cs[0][k].cuda() for k in ("y", "h", "post_w", "pre_w", "gate", "gate_ids")}
    h_out, x = torch.empty_like(b["h"]), torch.empty_like(b["y"])

    def call():
        sp.block_norm(b["y"], b["h"], h_out, x, post_w=b["post_w"], pre_w=b["pre_w"], gate=b["gate"],
                      gate_ids=b["gate_ids"], gate_kind="tanh")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for s in (1, 2, 0, 1):
        for k, t in b.items():
            t.copy_(cs[s][k])
        graph.replay()
        torch.cuda.synchronize()
        _check(cs[s], h_out.double().cpu().numpy(), x.double().cpu().numpy())


def test_a_block_of_both():
    """One transformer block as it is served: projections with adapters and the
    norms between them, captured once and replayed, against the eager calls and
    the oracle along the chain (each call against its stored inputs)."""
    from paper_2606_11244_amd import spear as sp
    from test_gpu_adapters import Slots
    from gpu_util import assert_parity
    M, D, F, dt = 12, 512, 1408, S.F16

    def layer(N, K, seed):
        L = S.make_layer(M=M, N=N, K=K, group_size=128, rank=0, act_dtype=dt, seed=seed)
        dl = sp.DeviceLayer(L)
        s = Slots(M, N, K, 5, 16, dt, seed=seed)
        return dict(dl.member(dl.problem(), with_ec=False), adapters=s.device(), L=L, s=s)
    q, k, v, o = (layer(n, D, i) for i, n in enumerate((D, 128, 128, D)))
    gate, up, down = layer(F, D, 4), layer(F, D, 5), layer(D, F, 6)
    x = q["x"]
    k["x"], v["x"] = x, x
    h = torch.randn(M, D, device="cuda").half()
    h1, x1, h2, x2 = (torch.empty(M, D, dtype=torch.float16, device="cuda") for _ in range(4))
    gate["x"], up["x"] = x1, x1
    w = [(1 + 0.1 * torch.randn(D, device="cuda")).half() for _ in range(4)]
    need = max(sp.adapters_workspace(g) for g in ([q, k, v], [o], [gate, up], [down]))
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")

    def single(m):
        sp.w4ec_linear_adapters(m["prob"], m["x"], m["qweight"], m["scales"], m["zeros"], m["adapters"], m["y"],
                                workspace=ws)

    def block():
        sp.w4ec_linear_adapters_group([q, k, v], ws)
        single(o)
        sp.block_norm(o["y"], h, h1, x1, post_w=w[0], pre_w=w[1])
        sp.w4ec_linear_adapters_group([gate, up], ws)
        single(down)
        sp.block_norm(down["y"], h1, h2, x2, post_w=w[2], pre_w=w[3], branch_scale=0.5)
    log("block of adapters and norms")
    block()
    torch.cuda.synchronize()
    outs = [m["y"] for m in (q, k, v, o, gate, up, down)] + [h1, x1, h2, x2]
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for _ in range(3):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for t, e in zip(outs, want):
            assert torch.equal(t, e)
    for m in (q, k, v, o, gate, up, down):
        xin = m["x"].double().cpu().numpy()
        L = m["L"]
        ref = O.w4_linear(xin, O.dequant(L.qweight, L.scales, L.zeros, L.group_size)) + m["s"].term(xin)
        assert_parity(m["y"].double().cpu().numpy(), ref, "block")
    for y, hin, hn, xn, i, beta in ((o["y"], h, h1, x1, 0, 1.0), (down["y"], h1, h2, x2, 2, 0.5)):
        c = dict(M=M, N=D, dt=torch.float16, f32=False, kind="mul", rho=1.0, beta=beta, off=0.0, eps=1e-5, y=y.cpu(),
                 h=hin.cpu(), post_w=w[i].cpu(), pre_w=w[i + 1].cpu(), gate=None, gate_ids=None)
        _check(c, hn.double().cpu().numpy(), xn.double().cpu().numpy())


@pytest.mark.parametrize("N", [264, 5003])
@pytest.mark.parametrize("f32", [False, True])
def test_rows_past_32_bits(N, f32):
    """The last rows lie past 2^32 bytes: the same values as dense rows."""
    from paper_2606_11244_amd import spear as sp
    M, ld = 5, (1 << 29) + 8
    g = torch.Generator().manual_seed(N)
    y, h = (torch.randn(M, N, generator=g).half().cuda() for _ in range(2))
    w = torch.randn(N, generator=g).half().cuda()
    h = h.float() if f32 else h
    want, x = torch.empty_like(h), torch.empty_like(y)
    sp.block_norm(y, h, want, x, post_w=w, pre_w=w, stream_scale=0.5)

    def far(t):
        big = torch.empty((M - 1) * ld + N, dtype=t.dtype, device="cuda").as_strided((M, N), (ld, 1))
        return big.copy_(t)
    log(f"block norm rows past 32 bits N={N} f32={f32}")
    fy, fh, fx = far(y), far(h), far(torch.zeros_like(y))
    sp.block_norm(fy, fh, fh, fx, post_w=w, pre_w=w, stream_scale=0.5)
    torch.cuda.synchronize()
    assert torch.equal(fh, want) and torch.equal(fx, x) and torch.equal(fy, y)


def test_two_calls_at_once():
    """Two streams read the same input and weights."""
    from paper_2606_11244_amd import spear as sp
    y, h = torch.randn(300, 4096, device="cuda").half(), torch.randn(300, 4096, device="cuda").half()
    w = torch.randn(4096, device="cuda").half()
    outs = [(torch.empty_like(y), torch.empty_like(y)) for _ in range(3)]
    sp.block_norm(y, h, *outs[2], post_w=w, pre_w=w)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for st, o in zip(streams, outs):
            sp.block_norm(y, h, *o, post_w=w, pre_w=w, stream=st)
    torch.cuda.synchronize()
    for o in outs[:2]:
        assert torch.equal(o[0], outs[2][0]) and torch.equal(o[1], outs[2][1])


@pytest.mark.parametrize("M,N", [(256, 4096), (257, 4096), (300, 2064), (260, 5003), (3000, 8192), (513, 8200)])
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("f32", [False, True])
def test_more_rows_than_cus(M, N, dt, f32):
    """Rows of several chunks a thread, and workgroups that take several rows."""
    log(f"block norm M={M} N={N} dt={dt} f32={f32}")
    c = _case(M, N, dt, f32=f32, gates="ids", kind="sigmoid", rho=0.7, beta=-1.5, pad=0 if N % 8 else 8)
    _check(c, *_run(c))
