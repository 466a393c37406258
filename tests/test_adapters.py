"""Host-side tests of the adapters' entry points and of the norms around a
block: arguments are refused before any launch, workspaces are laid out after
the layer's own, and the oracle's functions agree with direct loops."""
from __future__ import annotations

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import spear_oracle as O
from paper_2606_11244_amd import spear as sp

# fake, distinct, 16-byte aligned addresses: every call below is rejected on
# the host before anything touches them
NAMES = ["x", "y", "q", "s", "z", "A", "B", "w", "W", "res", "nw", "yn", "aA", "aB", "ids", "ranks",
         "scale", "h", "ho", "pw", "g", "gi", "xo"]
ADDR = {k: 0x7D0000000000 + i * (1 << 32) for i, k in enumerate(NAMES)}
DATA_BASE = (128 + 1024) * 1024


def _a(k):
    return ADDR[k] if isinstance(k, str) else k


def _ad(L=4, r=8, A="aA", B="aB", sa=0, sb=0, ranks="ranks", scale="scale", ids="ids"):
    return sp.Adapters(L, r, _a(A), _a(B), sa, sb, _a(ranks), _a(scale), _a(ids))


def _call(ad, prob=None, y="y", ws="W", ws_bytes=1 << 31, tail=None, ec=True, x="x"):
    prob = prob or sp.problem(4, 256, 256, 0, sp.F16, 8)
    w = sp.W4(ADDR["q"], ADDR["s"], ADDR["z"])
    e = sp.EC(ADDR["A"], ADDR["B"], 1.0, ADDR["w"], 0.0, None, None, None, None, 0, None, None)
    return sp.LIB.spear_w4ec_linear_adapters(
        ctypes.byref(prob), _a(x), ctypes.byref(w), ctypes.byref(e) if ec else None,
        ctypes.byref(ad) if ad is not None else None, ctypes.byref(tail) if tail else None, _a(y),
        _a(ws), ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(A=None), -1), (dict(B=None), -1), (dict(ids=None), -1),
    (dict(A=ADDR["aA"] + 8), -4), (dict(B=ADDR["aB"] + 2), -4), (dict(ids=ADDR["ids"] + 4), -4),
    (dict(ranks=ADDR["ranks"] + 4), -4), (dict(scale=ADDR["scale"] + 8), -4),
    (dict(L=-1), -2), (dict(r=-1), -2), (dict(r=257), -2),
    (dict(sa=8 * 256 - 8), -2), (dict(sb=8 * 256 - 1), -2), (dict(sa=8 * 256 + 4), -4),
    (dict(sa=1 << 31), -2), (dict(sb=-8), -2),
    (dict(A=ADDR["y"] + 16), -8), (dict(B=ADDR["y"] + 1024), -8), (dict(ids=ADDR["y"]), -8),
    (dict(ranks=ADDR["y"] + 16), -8), (dict(scale=ADDR["y"] + 16), -8),
    (dict(A=ADDR["y"] - 3 * 2 * 8 * 256), -8),  # the last slot reaches y
])
def test_adapters_refused(kw, code):
    assert _call(_ad(**kw)) == code


def test_adapters_call_refused():
    ad = _ad()
    assert _call(None) == -1
    assert _call(ad, x=None) == -1
    assert _call(ad, y=ADDR["y"] + 8) == -4
    assert _call(ad, ws=None) == -5
    assert _call(ad, ws=ADDR["W"] + 8) == -4
    assert _call(ad, y=ADDR["W"] + DATA_BASE) == -8
    assert _call(ad, prob=sp.problem(4, 256, 100, 0, sp.F16, 8)) == -2
    assert _call(ad, prob=sp.problem(4, 256, 256, 0, 2, 8)) == -3
    for ec in (True, False):
        assert _call(ad, tail=sp.Tail(_a("res"), _a("nw"), -1.0, _a("yn")), ec=ec) == -2
        assert _call(ad, tail=sp.Tail(_a("res"), _a("nw"), 1e-5, None), ec=ec) == -1
        assert _call(ad, tail=sp.Tail(_a("res"), _a("nw"), 1e-5, _a("aB")), ec=ec) == -8
        assert _call(ad, tail=sp.Tail(_a("res"), _a("nw"), 1e-5, ADDR["W"] + DATA_BASE), ec=ec) == -8
        assert _call(ad, tail=sp.Tail(ADDR["y"] + 16, None, 1e-5, None), ec=ec) == -8
    # products of 2^30 elements and more
    assert _call(_ad(r=256), prob=sp.problem(1, 1 << 22, 128, 0, sp.F16, 8)) == -2
    # an empty problem is a no-op
    assert _call(ad, prob=sp.problem(0, 256, 256, 0, sp.F16, 8), ws=None) == 0


def _members(*shapes, ec=True):
    out = []
    for M, N, K in shapes:
        t = torch.zeros(16)
        out.append(dict(prob=sp.problem(M, N, K, 0, sp.F16, 8), x=t, qweight=t, scales=t, zeros=t,
                        y=t, ec_args=dict(A=t, B=t, w_g=t) if ec else None))
    return out


def _group_ws(members, ads):
    arr, keep = sp._group_array(members)
    out = ctypes.c_size_t(0)
    ptrs = (ctypes.POINTER(sp.Adapters) * 4)(*[ctypes.pointer(a) if a else None for a in ads])
    st = sp.LIB.spear_adapters_workspace(len(members), arr, ptrs, ctypes.byref(out))
    return st, out.value


def test_workspace_follows_the_layers():
    ms = _members((4, 256, 256), (300, 512, 4096))
    base = sp.group_workspace(ms)
    st, none = _group_ws(ms, [None, None])
    assert (st, none) == (0, base)
    st, empty = _group_ws(ms, [_ad(L=0), _ad(r=0)])
    assert (st, empty) == (0, base)
    st, both = _group_ws(ms, [_ad(), _ad(r=64)])
    # at least the coordinates and the term of each, past the layers' data
    assert st == 0 and both >= max(base, DATA_BASE) + 4 * 8 * 4 + 4 * 256 * 2 + 300 * 64 * 4 + 300 * 512 * 2
    # a layer without data of its own: the adapters' lies past the counters
    one = _members((4, 256, 256), ec=False)
    assert sp.group_workspace(one) == DATA_BASE
    assert _group_ws(one, [_ad()])[1] > DATA_BASE
    assert _group_ws(ms, [_ad(L=-1), None])[0] == -2
    arr, keep = sp._group_array(ms)
    out = ctypes.c_size_t(0)
    assert sp.LIB.spear_adapters_workspace(2, arr, None, ctypes.byref(out)) == -1
    ptrs = (ctypes.POINTER(sp.Adapters) * 4)()
    assert sp.LIB.spear_adapters_workspace(2, arr, ptrs, None) == -1
    assert sp.LIB.spear_adapters_workspace(0, arr, ptrs, ctypes.byref(out)) == -2
    assert sp.LIB.spear_adapters_workspace(5, arr, ptrs, ctypes.byref(out)) == -2


def _group_call(specs, ads, ws_bytes=1 << 31):
    """specs: per member (y address, M)"""
    n = len(specs)
    arr = (sp.LayerCall * n)()
    keep = []
    for i, (y, M) in enumerate(specs):
        p = sp.problem(M, 256, 256, 0, sp.F16, 8)
        w = sp.W4(ADDR["q"], ADDR["s"], ADDR["z"])
        keep += [p, w]
        arr[i].prob, arr[i].w, arr[i].x, arr[i].y = ctypes.pointer(p), ctypes.pointer(w), ADDR["x"], y
    ptrs = (ctypes.POINTER(sp.Adapters) * n)(*[ctypes.pointer(a) if a else None for a in ads])
    return sp.LIB.spear_w4ec_linear_adapters_group(n, arr, ptrs, ADDR["W"], ws_bytes, None)


def test_group_refused():
    y0, y1 = ADDR["y"], ADDR["res"]
    arr = (sp.LayerCall * 1)()
    assert sp.LIB.spear_w4ec_linear_adapters_group(1, arr, None, ADDR["W"], 1 << 30, None) == -1
    assert _group_call([(y0, 4), (y1, 4)], [_ad(), _ad(ids=None)]) == -1
    assert _group_call([(y0, 4), (y1, 4)], [_ad(A=ADDR["aA"] + 8), None]) == -4
    assert _group_call([(y0, 4), (y1, 4)], [_ad(), _ad(r=300)]) == -2
    assert _group_call([(y0, 4), (y1, 4)], [_ad(), None], ws_bytes=4096) == -5
    # one member's output on another's adapters
    assert _group_call([(y0, 4), (y1, 4)], [_ad(), _ad(B=y0 + 32)]) == -8
    assert _group_call([(ADDR["W"] + DATA_BASE, 4), (y1, 4)], [_ad(), None]) == -8
    # empty members: nothing to do, nothing checked
    assert _group_call([(y0, 0), (y1, 0)], [_ad(), _ad(ids=None)]) == 0


def _norm(M=4, N=64, dt=sp.F16, stm=0, y="y", pw="pw", g="g", gi="gi", h="h", ho="ho", nw="nw", x="xo",
          lds=(0, 0, 0, 0, 0), n_gates=3, kind=0, rho=1.0, beta=1.0, off=0.0, eps=1e-5):
    return sp.BlockNorm(M, N, dt, stm, _a(y), _a(pw), _a(g), _a(gi), _a(h), _a(ho), _a(nw), _a(x),
                        *lds, n_gates, kind, rho, beta, off, eps)


@pytest.mark.parametrize("kw,code", [
    (dict(M=-1), -2), (dict(N=-1), -2), (dict(M=1 << 31), -2), (dict(N=1 << 30), -2),
    (dict(dt=2), -3), (dict(stm=2), -3), (dict(kind=3), -6), (dict(kind=-1), -6),
    (dict(eps=-1.0), -2), (dict(eps=math.nan), -2), (dict(rho=math.inf), -2), (dict(beta=math.nan), -2),
    (dict(off=math.inf), -2), (dict(lds=(63, 0, 0, 0, 0)), -2), (dict(lds=(0, 8, 0, 0, 0)), -2),
    (dict(lds=(0, 0, -64, 0, 0)), -2), (dict(lds=(0, 0, 0, 1 << 30, 0)), -2), (dict(lds=(0, 0, 0, 0, 1)), -2),
    (dict(n_gates=0), -2), (dict(gi=None, n_gates=3), -2), (dict(gi=None, n_gates=-1), -2),
    (dict(y=None), -1), (dict(ho=None), -1), (dict(x=None), -1),
    (dict(y=ADDR["y"] + 2), -4), (dict(h=ADDR["h"] + 8), -4), (dict(x=ADDR["xo"] + 8), -4),
    (dict(g=ADDR["g"] + 2), -4), (dict(gi=ADDR["gi"] + 4), -4), (dict(pw=ADDR["pw"] + 2), -4),
    (dict(nw=ADDR["nw"] + 2), -4), (dict(ho=ADDR["ho"] + 4), -4),
    (dict(ho="y"), -8), (dict(ho=ADDR["h"] + 16), -8), (dict(ho="h", lds=(0, 0, 0, 72, 0)), -8),
    (dict(x="y"), -8), (dict(x="h"), -8), (dict(x="ho"), -8), (dict(x=ADDR["nw"] + 16), -8),
    (dict(ho=ADDR["g"] + 3 * 128 - 16), -8), (dict(x=ADDR["gi"]), -8), (dict(ho="pw"), -8),
    (dict(y=ADDR["xo"] - 3 * 80 * 2, lds=(80, 0, 0, 0, 0)), -8),  # y's last row reaches x
])
def test_block_norm_refused(kw, code):
    a = _norm(**kw)
    assert sp.LIB.spear_block_norm(ctypes.byref(a), None) == code


def test_block_norm_empty_and_null():
    assert sp.LIB.spear_block_norm(None, None) == -1
    for kw in (dict(M=0, gi=None, n_gates=1), dict(N=0), dict(M=0, y=None, ho=None)):
        assert sp.LIB.spear_block_norm(ctypes.byref(_norm(**kw)), None) == 0


def test_binding_refuses_what_the_library_cannot_see():
    A, B = torch.zeros(3, 8, 256, dtype=torch.float16), torch.zeros(3, 64, 8, dtype=torch.float16)
    ids = torch.zeros(5, dtype=torch.int32)
    with pytest.raises(ValueError):
        sp.adapters(A, B[:2], ids)
    with pytest.raises(ValueError):
        sp.adapters(A, B[:, :, :4], ids)
    with pytest.raises(ValueError):
        sp.adapters(A.transpose(1, 2), torch.zeros(3, 64, 256, dtype=torch.float16), ids)
    with pytest.raises(TypeError):
        sp.adapters(A, B, ids.long())
    with pytest.raises(TypeError):
        sp.adapters(A, B.bfloat16(), ids)
    with pytest.raises(TypeError):
        sp.adapters(A, B, ids, scale=torch.ones(3, dtype=torch.float64))
    with pytest.raises(ValueError):
        sp.adapters(A, B, ids, ranks=torch.zeros(2, dtype=torch.int32))
    a = sp.adapters(A, B, ids)
    assert (a.n_adapters, a.rank, a.a_stride, a.b_stride) == (3, 8, 8 * 256, 8 * 64)
    wide = torch.zeros(3, 2, 8, 256, dtype=torch.float16)
    assert sp.adapters(wide[:, 1], B, ids).a_stride == 2 * 8 * 256
    # tensors in host memory are never handed to a kernel
    x = torch.zeros(5, 256, dtype=torch.float16)
    t = torch.zeros(16)
    with pytest.raises(ValueError):
        sp.w4ec_linear_adapters(sp.problem(5, 64, 256), x, t, t, t, a, t)
    with pytest.raises(ValueError):
        sp.block_norm(x, x, x.clone(), None)


def test_binding_refuses_overlapping_slots_and_rows():
    """Strides of zero (an expanded tensor) mean dense to the library."""
    A, B = torch.zeros(1, 8, 256, dtype=torch.float16), torch.zeros(3, 64, 8, dtype=torch.float16)
    ids = torch.zeros(5, dtype=torch.int32)
    with pytest.raises(ValueError, match="overlap"):
        sp.adapters(A.expand(3, 8, 256), B, ids)
    with pytest.raises(ValueError, match="overlap"):
        sp.adapters(A.repeat(3, 1, 1), B[:1].expand(3, 64, 8), ids)
    flat = torch.zeros(8 * 256 * 3, dtype=torch.float16)
    with pytest.raises(ValueError, match="overlap"):
        sp.adapters(flat.as_strided((3, 8, 256), (256, 256, 1)), B, ids)
    sp.adapters(A, B[:1], ids)
    rows = torch.zeros(1, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="overlap"):
        sp._rows(rows.expand(4, 64), (4, 64), torch.float16, "y")
    with pytest.raises(ValueError, match="overlap"):
        sp._rows(flat.as_strided((4, 64), (8, 1)), (4, 64), torch.float16, "h_out")
    assert sp._rows(rows, (1, 64), torch.float16, "y") == 0
    assert sp._rows(flat.as_strided((4, 64), (80, 1)), (4, 64), torch.float16, "y") == 80


def test_products_past_32_bits_refused():
    big = sp.problem(1 << 21, 128, 256)
    assert _call(_ad(r=256), prob=big, ec=False) == -2  # 2^21 tokens, 256 ranks
    assert _call(_ad(r=224), prob=big, ec=False, ws=None) == -5  # fits: the workspace is asked for
    assert _call(_ad(r=256), prob=sp.problem(1, 1 << 22, 128), ec=False) == -2
    assert _call(_ad(r=256), prob=sp.problem(1, 16, 1 << 22), ec=False) == -2


def test_oracle_against_loops():
    rng = np.random.default_rng(0)
    x, A, B = rng.normal(size=(5, 6)), rng.normal(size=(3, 4, 6)), rng.normal(size=(3, 7, 4))
    ids, ranks, scale = [2, -1, 0, 2, 3], [4, 1, 9], [0.5, 2.0, 1.5]
    got = O.adapters_term(x, A, B, ids, ranks, scale)
    for m, a in enumerate(ids):
        for n in range(7):
            want = 0.0
            if 0 <= a < 3:
                for j in range(min(ranks[a], 4)):
                    want += scale[a] * B[a, n, j] * sum(A[a, j, k] * x[m, k] for k in range(6))
            assert abs(got[m, n] - want) < 1e-12
    y, h, w, g = rng.normal(size=(4, 6)), rng.normal(size=(4, 6)), rng.normal(size=6), rng.normal(size=(2, 6))
    got = O.block_stream(y, h, w, g, [1, 5, 0, 1], "tanh", 0.5, 2.0, 1e-3, 1.0)
    for m, i in enumerate([1, 5, 0, 1]):
        rms = math.sqrt(sum(v * v for v in y[m]) / 6 + 1e-3)
        for n in range(6):
            gate = math.tanh(g[i, n]) if i < 2 else 1.0
            assert abs(got[m, n] - (0.5 * h[m, n] + 2.0 * gate * y[m, n] / rms * (1.0 + w[n]))) < 1e-12
