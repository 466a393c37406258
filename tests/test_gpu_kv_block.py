"""Attention over the cache between the layers that it stands between: the grouped
4-bit q, k and v projections, rotary positions with the cache's writing, attention,
and the output projection, one after another on one stream and in a captured graph;
every stage against its reference on what it was given."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv_util as U
from gpu_util import assert_parity, with_fields
from oracle import spear_oracle as O
from paper_2606_11244_amd import synth as S
from test_gpu_kv import Server

pytestmark = pytest.mark.gpu


def _bits(t):
    return np.ascontiguousarray(t.cpu().view(torch.int16).numpy()).view(np.uint16)


class Block:
    """The four projections of one attention block for T tokens, and the server's step between them."""

    def __init__(self, server, T, hidden, act, seed):
        from paper_2606_11244_amd import spear as sp
        self.sp, self.s = sp, server
        dt = S.BF16 if act is torch.bfloat16 else S.F16
        cache = server.caches[0]
        H, kvh, D = server.x[0][0].shape[1], cache.kv_heads, cache.head_dim
        sizes = [(H * D, hidden), (kvh * D, hidden), (kvh * D, hidden), (hidden, H * D)]
        self.layers = [S.make_layer(M=T, N=n, K=k, group_size=128, rank=16, act_dtype=dt, seed=seed, module_id=i, w_std=0.08)
                       for i, (n, k) in enumerate(sizes)]
        self.dev = [sp.DeviceLayer(L) for L in self.layers]
        self.x = self.dev[0].x
        for d in self.dev[1:3]:
            d.x = self.x
        self.q, self.k, self.v = (d.y.view(T, h, D) for d, h in zip(self.dev, (H, kvh, kvh)))
        self.qr, self.out = torch.zeros_like(self.q), torch.zeros_like(self.q)
        self.dev[3].x = self.out.view(T, H * D)
        probs = [d.problem() for d in self.dev]
        self.members = [d.member(p, with_ec=True) for d, p in zip(self.dev[:3], probs)]
        self.group_ws = torch.zeros(max(256, sp.group_workspace(self.members)), dtype=torch.uint8, device="cuda")
        self.o_prob, self.o_ws = probs[3], sp.allocate_workspace(probs[3], True)
        server.caches, server.qr = server.caches[:1], [self.qr]

    def step(self):
        s, kv = self.s, self.s.kv
        self.sp.w4ec_linear_group(self.members, self.group_ws)
        kv.pages(s.batch, s.held, s.fresh, s.free, s.slots, s.positions, s.taken, page_tokens=s.P)
        kv.attention_plan(s.plan)
        kv.append(s.caches[0], self.k, self.v, s.slots, s.positions, rope=s.rope, q=self.q, q_out=self.qr)
        kv.attention(s.plan, self.qr, self.out, workspace=s.ws, cache=s.caches[0])
        self.dev[3].run_ec(self.o_prob, self.o_ws)

    def feed(self, fresh, seed):
        s = self.s
        s.fresh.copy_(torch.tensor(fresh, dtype=torch.int32))
        self.x.copy_(torch.randn(self.x.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
        # rows behind the last request are left as they were: those of before, and what the server's check looks for
        self.out.fill_(9.0)
        self.qr.zero_()
        s.out = [self.out]

    def check(self):
        for L, d in zip(self.layers[:3], self.dev):
            assert_parity(d.y.float().cpu().numpy().astype(np.float64), O.w4ec_linear(with_fields(L, x=_bits(self.x))))
        s, n = self.s, int(self.s.batch.starts[-1])
        freqs = [f % 2 ** 64 for f in s.rope.freqs.tolist()]
        q = self.q.cpu()[:n]
        want = U.turned(q, s.positions.tolist()[:n], freqs, s.rope.c.rotary_dim, False, 1.0)
        # an fp32 rotation is off by 2^-21 of the pair's length at most, and rounded once
        room = U.U[s.act] * want.abs() + q.double().abs().amax(dim=2, keepdim=True) * 2 ** -20 + 2.0 ** -25
        assert bool(((self.qr.cpu()[:n].double() - want).abs() <= room).all())
        s.check()
        L = with_fields(self.layers[3], x=_bits(self.dev[3].x))
        assert_parity(self.dev[3].y.float().cpu().numpy().astype(np.float64), O.w4ec_linear(L))


@pytest.mark.parametrize("act,codes", [(torch.float16, torch.int8), (torch.bfloat16, torch.float8_e4m3fn)])
def test_a_blocks_projections_and_attention(act, codes):
    s = Server(4, 75, 60, heads=8, kvh=2, D=64, P=16, act=act, codes=codes)
    b = Block(s, 75, 512, act, 1)
    for i, fresh in enumerate(([60, 1, 9, 0], [1, 50, 1, 20], [1, 1, 1, 1])):
        b.feed(fresh, i)
        b.step()
        b.check()
        s.advance()


@pytest.mark.parametrize("act,codes", [(torch.float16, torch.float8_e4m3fn), (torch.bfloat16, torch.int8)])
def test_a_blocks_decoding_step_in_a_graph(act, codes):
    s = Server(4, 4, 1, heads=8, kvh=2, D=128, P=32, act=act, codes=codes)
    b = Block(s, 4, 512, act, 2)
    b.feed([1, 1, 1, 1], 0)
    b.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for i in range(5):
        b.feed([1, i % 2, 1, 1], 10 + i)
        graph.replay()
        torch.cuda.synchronize()
        b.check()
        s.advance()
        torch.randn(1000, device="cuda").sum().item()
