"""What is timed of the operators beside the 4-bit linear layer: low-rank
adapters of many requests at once, and the norms around a block.

Kinds of case:

* "linear": one 4-bit projection (with the EC where `ec` is a rank) and the
  adapters of its tokens: y[m] = W x[m] (+ EC) + s_a B_a (A_a x[m]) for the
  token's adapter a = ids[m], nothing for a token without one; with `tail` the
  residual and the next RMSNorm as well.
* "group": projections of one hidden state (q, k, v; gate, up) as one grouped
  call, each with adapters of its own.
* "norm": h' = rho h + beta gate (.) RMSNorm(y; w_post), x = RMSNorm(h'; w_pre):
  the norms after a block and before the next one, its gate and its residual.
* "block": a transformer block of these: q, k, v; o; norms; gate, up on the
  norms' output; down; norms (attention and the activation between the
  projections are not part of it, so o and down have inputs of their own).

Shapes are the Llama-3.2-1B, Llama-3-8B and Llama-2-70B layers that this
repository serves, one of eight tensor-parallel shards, and generic ones.
Weights are N(0, 0.02) quantised round-to-nearest to 4 bits, activations
N(0, 1), adapter factors N(0, 0.02), EC factors N(0, 0.01).
"""
import math

import torch

own = False

_DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_CODE = {"f16": 0, "bf16": 1, "f32": 2}
_EPS = 1e-5
_B_G, _ALPHA = 0.1, 1.0


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _adapted(kind, M, K, Ns, *, dtype="f16", group=128, slots=16, used=4, rank=16, mixed=False,
             runs=False, bare=0, ec=0, tail=False, name=None):
    c = dict(kind=kind, M=M, K=K, Ns=",".join(str(n) for n in Ns), dtype=dtype, group=group,
             slots=slots, used=used, rank=rank, mixed=mixed, runs=runs, bare=bare, ec=ec, tail=tail)
    return dict(c, name=name) if name else c


def _norm(M, N, *, dtype="f16", stream="act", post=True, pre=True, gates="one", gate="mul",
          rho=1.0, beta=1.0, name=None):
    c = dict(kind="norm", M=M, N=N, dtype=dtype, stream=stream, post=post, pre=pre, gates=gates,
             gate=gate, rho=rho, beta=beta)
    return dict(c, name=name) if name else c


def _block(M, D, KV, F, *, dtype="f16", group=128, slots=16, used=4, rank=16, runs=False, name=None):
    c = dict(kind="block", M=M, D=D, KV=KV, F=F, dtype=dtype, group=group, slots=slots, used=used,
             rank=rank, mixed=False, runs=runs, bare=0)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one request on the small model, one projection: nothing but latency
        _adapted("linear", 1, 2048, [2048], slots=8, used=1, rank=8, name="1b q, 1 token"),
        # sixteen requests decoding with an adapter each: q, k, v of the 8B model
        _adapted("group", 16, 4096, [4096, 1024, 1024], dtype="bf16", group=0, slots=32, used=16,
                 name="8b qkv, 16 requests"),
        # a shard of the headline model with its EC: 48 tokens, adapters of several ranks, some
        # requests on the shared weights alone
        _adapted("linear", 48, 8192, [3584], slots=64, used=24, rank=64, mixed=True, bare=12, ec=64,
                 name="70b/8 gate, 48 tokens, ec"),
        # a chunk through a layer of no particular shape, with the residual and the next norm
        _adapted("linear", 77, 2944, [5000], dtype="bf16", slots=5, used=3, rank=24, runs=True,
                 tail=True, name="ragged 77, tail"),
        # prompts of four requests in one chunk, down projection with the tail
        _adapted("linear", 300, 14336, [4096], dtype="bf16", group=0, slots=8, used=4, rank=32,
                 runs=True, tail=True, name="8b down, 300 tokens"),
        # long prompts of eight requests: gate and up of the 8B model
        _adapted("group", 2048, 4096, [14336, 14336], slots=16, used=8, rank=32, runs=True,
                 name="8b gate up, 2048 tokens"),
        # long prompts on the headline model
        _adapted("linear", 4096, 8192, [8192], slots=16, used=6, runs=True, name="70b q, 4096 tokens"),
        # the norms of one token
        _norm(1, 4096, name="norms, 1 token"),
        # a decode batch whose residual stream is held in 32 bits, a gate row for each request
        _norm(24, 8192, dtype="bf16", stream="f32", gates="ids", gate="tanh", rho=0.9, beta=1.2,
              name="norms, 24 x 8192, 32 bits"),
        # rows of odd length
        _norm(301, 5003, dtype="bf16", gates="none", name="norms, 301 x 5003"),
        # a long prompt
        _norm(4096, 8192, gates="row", gate="sigmoid", name="norms, 4096 x 8192"),
        # one block of the 8B model, eight requests decoding
        _block(8, 4096, 1024, 14336, used=8, name="8b block, 8 requests"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(("f16", "bf16"))
    kind = rng.choice(("linear", "linear", "group", "norm", "norm", "block"))
    if kind == "norm":
        M, N = _log_uniform(rng, 1, 4096), _log_uniform(rng, 64, 8192)
        if rng.random() < 0.5:
            N = max(8, N // 8 * 8)
        return _norm(M, N, dtype=dtype, stream=rng.choice(("act", "act", "f32")),
                     post=rng.random() < 0.8, pre=rng.random() < 0.9,
                     gates=rng.choice(("none", "one", "row", "ids")),
                     gate=rng.choice(("mul", "tanh", "sigmoid")), rho=round(rng.uniform(0.5, 1.5), 3),
                     beta=round(rng.uniform(0.5, 1.5), 3))
    M = _log_uniform(rng, 1, 2048)
    slots = _log_uniform(rng, 1, 64)
    opt = dict(dtype=dtype, group=rng.choice((128, 128, 0)), slots=slots,
               used=max(1, min(slots, M, _log_uniform(rng, 1, 64))),
               rank=rng.choice((4, 8, 16, 16, 24, 32, 64)), runs=M > 64 or rng.random() < 0.3)
    if kind == "block":
        D, KV, F = rng.choice(((2048, 512, 8192), (4096, 1024, 14336)))
        return _block(min(M, 512), D, KV, F, **dict(opt, used=min(opt["used"], M, 512)))
    K = 128 * _log_uniform(rng, 4, 64)
    Ns = [_log_uniform(rng, 200, 8192) for _ in range(1 if kind == "linear" else rng.choice((2, 3)))]
    bare = rng.choice((0, 0, M // 4))
    return _adapted(kind, M, K, Ns, **dict(opt, used=max(1, min(opt["used"], M - bare))),
                    mixed=rng.random() < 0.4, bare=bare,
                    ec=rng.choice((0, 0, 16, 32)) if kind == "linear" else 0,
                    tail=kind == "linear" and rng.random() < 0.4)


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


def _randn(g, std, *shape):
    return torch.randn(shape, device="cuda", generator=g) * std


def _weight(case, g, N, K):
    """4-bit codes packed eight to a word (lowest first), scales as fp16, zero points."""
    G = K if case["group"] == 0 else case["group"]
    w = _randn(g, 0.02, N, K // G, G)
    lo, hi = w.amin(dim=2, keepdim=True), w.amax(dim=2, keepdim=True)
    s = ((hi - lo) / 15.0).half()
    z = torch.clamp(torch.round(-lo / s.float()), 0, 15)
    q = torch.clamp(torch.round(w / s.float()) + z, 0, 15).to(torch.uint8).view(N, K)
    words = (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous().view(torch.int32)
    return dict(qweight=words, scales=s.view(N, K // G), zeros=z.to(torch.uint8).view(N, K // G))


def _slot_ranks(case):
    """The ranks of the used adapters, in the order in which tokens meet them."""
    return [max(1, case["rank"] >> (i % 3)) if case["mixed"] else case["rank"]
            for i in range(case["used"])]


def _ids(case, g):
    """Which slot each token takes (-1: none), and each slot's rank. Tokens meet the used slots in
    runs (prompts) or in turn (decoding requests); slots and bare tokens are the seed's choice."""
    M, used = case["M"], case["used"]
    slots = torch.randperm(case["slots"], device="cuda", generator=g)[:used]
    t = torch.arange(M - case["bare"], device="cuda")
    turn = t * used // max(1, t.numel()) if case["runs"] else t % used
    ids = torch.full((M,), -1, dtype=torch.int64, device="cuda")
    place = torch.randperm(M, device="cuda", generator=g)[case["bare"]:].sort().values
    ids[place] = slots[turn]
    ranks = torch.full((case["slots"],), case["rank"], dtype=torch.int32, device="cuda")
    ranks[slots] = torch.tensor(_slot_ranks(case), dtype=torch.int32, device="cuda")
    return ids.to(torch.int32), ranks


def _module(case, seed, i, N, K, ec, tail, ids, ranks):
    g, dt = _generator(seed, 1, i), _DT[case["dtype"]]
    M, L, R = case["M"], case["slots"], case["rank"]
    m = dict(N=N, K=K, M=M, **_weight(case, g, N, K))
    m["A"] = _randn(g, 0.02, L, R, K).to(dt)
    m["B"] = _randn(g, 0.02, L, N, R).to(dt)
    m["scale"] = 0.5 + torch.rand(L, device="cuda", generator=g)
    m["ids"], m["ranks"] = ids, ranks
    if ec:
        m["ec"] = dict(A=_randn(g, 0.01, ec, K).to(dt), B=_randn(g, 0.01, N, ec).to(dt),
                       w_g=_randn(g, 0.05, K).to(dt))
    if tail:
        m["residual"] = _randn(g, 1.0, M, N).to(dt)
        m["norm_w"] = (1.0 + _randn(g, 0.1, N)).to(dt)
    return m


def _norm_inputs(case, g, M, N, y):
    dt = _DT[case["dtype"]]
    n = dict(M=M, N=N, y=y, rho=case["rho"], beta=case["beta"], gate_kind=case["gate"])
    n["h"] = _randn(g, 1.0, M, N).to(dt if case["stream"] == "act" else torch.float32)
    n["post_w"] = (1.0 + _randn(g, 0.1, N)).to(dt) if case["post"] else None
    n["pre_w"] = (1.0 + _randn(g, 0.1, N)).to(dt) if case["pre"] else None
    rows = {"none": 0, "one": 1, "row": M, "ids": max(1, M // 3)}[case["gates"]]
    n["gate"] = _randn(g, 1.0, rows, N).to(dt) if rows else None
    n["gate_ids"] = None
    if case["gates"] == "ids":
        n["gate_ids"] = torch.randint(0, rows, (M,), device="cuda", generator=g, dtype=torch.int32)
    return n


_BLOCK_NORM = dict(stream="act", post=True, pre=True, gates="one", gate="mul", rho=1.0, beta=1.0)


def _modules(case):
    """(N, K, EC rank, tail) of each projection, in call order."""
    if case["kind"] == "block":
        D, KV, F = case["D"], case["KV"], case["F"]
        return [(D, D, 0, False), (KV, D, 0, False), (KV, D, 0, False), (D, D, 0, False),
                (F, D, 0, False), (F, D, 0, False), (D, F, 0, False)]
    return [(int(n), case["K"], case["ec"], case["tail"]) for n in case["Ns"].split(",")]


def _inputs(case, seed):
    """Everything that a pass reads, by the seed alone."""
    g, dt, M = _generator(seed, 2), _DT[case["dtype"]], case["M"]
    if case["kind"] == "norm":
        return dict(norm=_norm_inputs(case, g, M, case["N"], (_randn(g, 1.0, M, case["N"]) * 3.0).to(dt)))
    ids, ranks = _ids(case, g)
    mods = [_module(case, seed, i, *m, ids, ranks) for i, m in enumerate(_modules(case))]
    st = dict(mods=mods, x=_randn(g, 1.0, M, mods[0]["K"]).to(dt))
    if case["kind"] == "block":
        D, F = case["D"], case["F"]
        st["x_o"], st["x_down"] = _randn(g, 1.0, M, D).to(dt), _randn(g, 1.0, M, F).to(dt)
        c = dict(case, **_BLOCK_NORM)
        st["n1"], st["n2"] = (_norm_inputs(c, g, M, D, None) for _ in range(2))
    return st


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    if own:
        _keep(st)
    return st


def _keep(st):
    """What a program keeps beside its tensors: descriptions of the problems and of the adapters,
    output buffers and the workspace."""
    from paper_2606_11244_amd import spear as sp
    case = st["case"]
    dt, M = _DT[case["dtype"]], case["M"]
    st["sp"] = sp
    for n in (st[k] for k in ("norm", "n1", "n2") if k in st):
        n["h_out"] = torch.empty_like(n["h"])
        n["x"] = torch.empty((M, n["N"]), dtype=dt, device="cuda") if n["pre_w"] is not None else None
    if case["kind"] == "norm":
        return
    inputs = [st["x"]] * len(st["mods"])
    if case["kind"] == "block":
        x2 = st["n1"]["x"]
        inputs = [st["x"], st["x"], st["x"], st["x_o"], x2, x2, st["x_down"]]
    for m, x in zip(st["mods"], inputs):
        e = m.get("ec")
        m["prob"] = sp.problem(M, m["N"], m["K"], case["group"], _CODE[case["dtype"]],
                               e["A"].shape[0] if e else 0)
        m["x"], m["y"] = x, torch.empty((M, m["N"]), dtype=dt, device="cuda")
        m["y_norm"] = torch.empty_like(m["y"]) if "norm_w" in m else None
        m["ec_args"] = dict(e, b_g=_B_G, alpha=_ALPHA) if e else None
        m["adapters"] = sp.adapters(m["A"], m["B"], m["ids"], ranks=m["ranks"], scale=m["scale"])
    parts = [st["mods"]] if case["kind"] != "block" else [st["mods"][a:b] for a, b in ((0, 3), (3, 4), (4, 6), (6, 7))]
    need = max(sp.adapters_workspace(p) for p in parts)
    st["ws"] = torch.zeros(max(256, need), dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _formulas(state, torch.float32)


def _run_own(st):
    sp, case = st["sp"], st["case"]
    if case["kind"] == "norm":
        return _own_norm(sp, st["norm"], st["norm"]["y"])
    mods, ws = st["mods"], st["ws"]
    if case["kind"] == "group":
        sp.w4ec_linear_adapters_group(mods, ws)
        return [m["y"] for m in mods]
    if case["kind"] == "linear":
        _own_linear(sp, mods[0], ws)
        return [mods[0]["y"]] + ([mods[0]["y_norm"]] if mods[0]["y_norm"] is not None else [])
    sp.w4ec_linear_adapters_group(mods[0:3], ws)
    _own_linear(sp, mods[3], ws)
    o1 = _own_norm(sp, st["n1"], mods[3]["y"])
    sp.w4ec_linear_adapters_group(mods[4:6], ws)
    _own_linear(sp, mods[6], ws)
    o2 = _own_norm(sp, st["n2"], mods[6]["y"])
    return [m["y"] for m in mods] + o1 + o2


def _own_linear(sp, m, ws):
    sp.w4ec_linear_adapters(m["prob"], m["x"], m["qweight"], m["scales"], m["zeros"], m["adapters"],
                            m["y"], ec_args=m["ec_args"], residual=m.get("residual"),
                            norm_w=m.get("norm_w"), eps=_EPS, y_norm=m["y_norm"], workspace=ws)


def _own_norm(sp, n, y):
    sp.block_norm(y, n["h"], n["h_out"], n["x"], post_w=n["post_w"], pre_w=n["pre_w"],
                  gate=n["gate"], gate_ids=n["gate_ids"], gate_kind=n["gate_kind"],
                  stream_scale=n["rho"], branch_scale=n["beta"], eps=_EPS)
    return [n["h_out"]] + ([n["x"]] if n["x"] is not None else [])


def _plain_weight(m, t):
    N, K = m["N"], m["K"]
    shifts = torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)
    q = ((m["qweight"].view(N, K // 8, 1) >> shifts) & 15).view(N, m["scales"].shape[1], -1).to(t)
    return ((q - m["zeros"].to(t)[:, :, None]) * m["scales"].to(t)[:, :, None]).view(N, K)


def _plain_linear(m, x, t, dt):
    """y (and y_norm with a tail), from every slot's product and a mask of the token's own."""
    x = x.to(t)
    y = x @ _plain_weight(m, t).T
    if "ec" in m:
        e = {k: v.to(t) for k, v in m["ec"].items()}
        g = 1.0 / (1.0 + torch.exp(-(x @ e["w_g"] + _B_G)))
        y = y + _ALPHA * ((g[:, None] * (x @ e["A"].T)) @ e["B"].T)
    L, R, K = m["A"].shape
    u = (x @ m["A"].to(t).view(L * R, K).T).view(-1, L, R) * m["scale"].to(t)[None, :, None]
    slot = torch.arange(L, device="cuda")
    mine = (m["ids"][:, None] == slot[None, :])[:, :, None]
    live = torch.arange(R, device="cuda")[None, :] < m["ranks"][:, None]
    u = torch.where(mine & live[None], u, torch.zeros_like(u))
    y = y + u.reshape(-1, L * R) @ m["B"].to(t).permute(0, 2, 1).reshape(L * R, -1)
    if "residual" not in m:
        return [y.to(dt)]
    y = y + m["residual"].to(t)
    stored = y.to(dt).to(t)
    return [y.to(dt), (_plain_rms(stored) * m["norm_w"].to(t)).to(dt)]


def _plain_rms(v):
    return v / torch.sqrt((v * v).mean(dim=1, keepdim=True) + _EPS)


def _plain_norm(n, y, t, dt):
    o = y.to(t)
    if n["post_w"] is not None:
        o = _plain_rms(o) * n["post_w"].to(t)
    if n["gate"] is not None:
        gate = n["gate"].to(t)
        gate = gate[n["gate_ids"].long()] if n["gate_ids"] is not None else gate
        if n["gate_kind"] == "sigmoid":
            gate = 1.0 / (1.0 + torch.exp(-gate))
        elif n["gate_kind"] == "tanh":
            gate = 1.0 - 2.0 / (torch.exp(2.0 * gate) + 1.0)
        o = gate * o
    h = (n["rho"] * n["h"].to(t) + n["beta"] * o).to(n["h"].dtype)
    return [h] + ([(_plain_rms(h.to(t)) * n["pre_w"].to(t)).to(dt)] if n["pre_w"] is not None else [])


def _formulas(st, t):
    case = st["case"]
    dt = _DT[case["dtype"]]
    if case["kind"] == "norm":
        return _plain_norm(st["norm"], st["norm"]["y"], t, dt)
    mods, x = st["mods"], st["x"]
    if case["kind"] != "block":
        outs = [_plain_linear(m, x, t, dt) for m in mods]
        return [o for out in outs for o in out]
    q, k, v = (_plain_linear(m, x, t, dt)[0] for m in mods[0:3])
    o = _plain_linear(mods[3], st["x_o"], t, dt)[0]
    o1 = _plain_norm(st["n1"], o, t, dt)
    gate, up = (_plain_linear(m, o1[1], t, dt)[0] for m in mods[4:6])
    down = _plain_linear(mods[6], st["x_down"], t, dt)[0]
    return [q, k, v, o, gate, up, down] + o1 + _plain_norm(st["n2"], down, t, dt)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def _norm_work(M, N, case):
    rows = {"none": 0, "one": 1, "row": M, "ids": max(1, M // 3)}[case["gates"]]
    h = 4 if case["stream"] == "f32" else 2
    b = M * N * (2 + 2 * h) + 2 * rows * N + (4 * M if case["gates"] == "ids" else 0)
    b += 2 * N * (case["post"] + case["pre"]) + (2 * M * N if case["pre"] else 0)
    return b, M * N * (3 + 4 * case["post"] + 4 * case["pre"] + (1 if rows else 0))


def work(case):
    M, b, f = case["M"], 0, 0
    if case["kind"] == "norm":
        b, f = _norm_work(M, case["N"], case)
        return {"bytes": b, "flops": f}
    r_sum = sum(_slot_ranks(case))
    r_mean = r_sum * (M - case["bare"]) / case["used"]
    mods = _modules(case)
    for N, K, ec, tail in mods:
        G = K if case["group"] == 0 else case["group"]
        b += N * K // 2 + 3 * N * (K // G) + 2 * M * N + 2 * r_sum * (N + K)
        f += 2 * M * N * K + int(2 * r_mean * (N + K))
        if ec:
            b += 2 * ec * (N + K) + 2 * K
            f += 2 * M * ec * (N + K) + 2 * M * K
        if tail:
            b += 4 * M * N + 2 * N
            f += 6 * M * N
    b += 2 * M * mods[0][1] + 4 * M
    if case["kind"] == "block":
        nb, nf = _norm_work(M, case["D"], dict(case, **_BLOCK_NORM))
        # the input of gate and up, each norm's y: written by one call, read by the next
        b += 2 * M * (case["D"] + case["F"]) + 2 * nb - 2 * M * case["D"]
        f += 2 * nf
    return {"bytes": b, "flops": f}


# ---------------------------------------------------------------------------
# the operators' definition in 64 bits, token by token where adapters differ
# ---------------------------------------------------------------------------

def _exact_dense(m):
    N, K = m["N"], m["K"]
    b = m["qweight"].view(torch.uint8).view(N, K // 2)
    q = torch.stack((b & 15, b >> 4), dim=2).view(N, K).double()
    G = K // m["scales"].shape[1]
    s = m["scales"].double().repeat_interleave(G, dim=1)
    return (q - m["zeros"].double().repeat_interleave(G, dim=1)) * s


def _exact_linear(m, x):
    x = x.double()
    y = x @ _exact_dense(m).T
    if "ec" in m:
        e = m["ec"]
        gate = torch.sigmoid(x @ e["w_g"].double() + _B_G)
        y += _ALPHA * (gate[:, None] * (x @ e["A"].double().T)) @ e["B"].double().T
    for a in sorted(set(m["ids"].tolist()) - {-1}):
        rows = (m["ids"] == a).nonzero().squeeze(1)
        r = int(m["ranks"][a])
        u = x[rows] @ m["A"][a, :r].double().T
        y[rows] += float(m["scale"][a]) * (u @ m["B"][a, :, :r].double().T)
    if "residual" not in m:
        return [y]
    y += m["residual"].double()
    rms = torch.sqrt((y ** 2).sum(1, keepdim=True) / y.shape[1] + _EPS)
    return [y, y / rms * m["norm_w"].double()]


def _exact_norm(n, y):
    y = y.double()
    if n["post_w"] is not None:
        y = n["post_w"].double() * y * torch.rsqrt((y ** 2).sum(1, keepdim=True) / n["N"] + _EPS)
    if n["gate"] is not None:
        g = n["gate"].double()
        if n["gate_ids"] is not None:
            g = torch.stack([g[i] for i in n["gate_ids"].tolist()])
        y = y * {"mul": lambda v: v, "tanh": torch.tanh, "sigmoid": torch.sigmoid}[n["gate_kind"]](g)
    h = n["rho"] * n["h"].double() + n["beta"] * y
    if n["pre_w"] is None:
        return [h]
    return [h, n["pre_w"].double() * h * torch.rsqrt((h ** 2).sum(1, keepdim=True) / n["N"] + _EPS)]


def exact(case, seed):
    st = _inputs(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(st["norm"], st["norm"]["y"])
    mods = st["mods"]
    if case["kind"] != "block":
        return [o for m in mods for o in _exact_linear(m, st["x"])]
    q, k, v = (_exact_linear(m, st["x"])[0] for m in mods[0:3])
    o = _exact_linear(mods[3], st["x_o"])[0]
    o1 = _exact_norm(st["n1"], o)
    gate, up = (_exact_linear(m, o1[1])[0] for m in mods[4:6])
    down = _exact_linear(mods[6], st["x_down"])[0]
    return [q, k, v, o, gate, up, down] + o1 + _exact_norm(st["n2"], down)
