"""Python binding of the C ABI in include/spear_kv.h (argument marshalling
only): attention over a paged cache held in 8 bits, with the block tables, the
rotary positions and the cache's writing that go before it.

A step of a serving program:

    cache = Cache(k, v, k_scale, v_scale, torch.bfloat16)      # per layer, or new_cache(...)
    batch = Batch(table, tokens, max_new=1)
    plan = AttentionPlan(cache, batch, heads)
    work = torch.zeros(attention_workspace(plan), dtype=torch.uint8, device="cuda")

    pages(batch, held, fresh, free, slots, positions, taken, page_tokens=64)
    attention_plan(plan)                                       # once a step
    append(cache, k_new, v_new, slots, positions, rope=rope, q=q, q_out=q)
    attention(plan, q, out, workspace=work, cache=cache)       # per layer

Functions mirror the C entry points; shapes, types and errors are those of the
header. Every step runs in libspear.so's HIP kernels: there is no fallback.
"""
from __future__ import annotations

import ctypes

import torch

from .spear import LIB, SpearError, _device_of, _raw_stream

INT8, E4M3 = 0, 1
_CODES = {torch.int8: INT8, torch.float8_e4m3fn: E4M3}
_ACTS = {torch.float16: 0, torch.bfloat16: 1}
_i32, _i64, _p, _f = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float


class _Cache(ctypes.Structure):
    _fields_ = [("format", _i32), ("act_dtype", _i32), ("kv_heads", _i32), ("head_dim", _i32),
                ("page_tokens", _i32), ("reserved", _i32), ("pages", _i64), ("k", _p), ("v", _p),
                ("k_scale", _p), ("v_scale", _p)]


class _Batch(ctypes.Structure):
    _fields_ = [("requests", _i32), ("tokens", _i32), ("max_new", _i32), ("width", _i32),
                ("table_ld", _i32), ("reserved", _i32), ("starts", _p), ("lens", _p), ("table", _p)]


class _Pages(ctypes.Structure):
    _fields_ = [("page_tokens", _i32), ("n_free", _i32), ("held", _p), ("fresh", _p),
                ("free_pages", _p), ("slots", _p), ("positions", _p), ("taken", _p)]


class _Rope(ctypes.Structure):
    _fields_ = [("rotary_dim", _i32), ("interleaved", _i32), ("magnitude", _f), ("reserved", _i32),
                ("freqs", _p)]


class _Append(ctypes.Structure):
    _fields_ = [("tokens", _i32), ("heads", _i32), ("q", _p), ("k", _p), ("v", _p), ("q_out", _p),
                ("q_ld", _i64), ("k_ld", _i64), ("v_ld", _i64), ("q_out_ld", _i64), ("slots", _p),
                ("positions", _p), ("rope", _Rope)]


class _Attention(ctypes.Structure):
    _fields_ = [("cache", ctypes.POINTER(_Cache)), ("batch", ctypes.POINTER(_Batch)),
                ("heads", _i32), ("window", _i32), ("prefix", _p), ("plan", _p),
                ("plan_bytes", ctypes.c_size_t), ("q", _p), ("out", _p), ("q_ld", _i64),
                ("out_ld", _i64), ("slopes", _p), ("scale", _f), ("softcap", _f),
                ("workspace", _p), ("workspace_bytes", ctypes.c_size_t)]


LIB.spear_kv_pages.argtypes = [ctypes.POINTER(_Batch), ctypes.POINTER(_Pages), _p]
LIB.spear_rope_frequencies.argtypes = [_i32] + [ctypes.c_double] * 5 + [_p]
LIB.spear_kv_append.argtypes = [ctypes.POINTER(_Cache), ctypes.POINTER(_Append), _p]
LIB.spear_kv_read.argtypes = [ctypes.POINTER(_Cache), _i64, _p, _p, _p, _p]
LIB.spear_attention_sizes.argtypes = [ctypes.POINTER(_Attention)] + [ctypes.POINTER(ctypes.c_size_t)] * 2
LIB.spear_attention_plan.argtypes = [ctypes.POINTER(_Attention), _p]
LIB.spear_attention.argtypes = [ctypes.POINTER(_Attention), _p]


def _check(status, where):
    if status != 0:
        raise SpearError(status, where)


def _ints(t, n, what):
    if t.dtype is not torch.int32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} is [{n}] int32")
    return t.data_ptr()


def _size(v, what):
    """A size as the C structs hold it, which keep the lower 32 bits of any."""
    v = int(v)
    if not -(1 << 31) <= v < 1 << 31:
        raise ValueError(f"{what} is a number of 32 bits (got {v})")
    return v


def _on(holder, dev):
    """That a cache's, batch's or rotation's tensors are on GPU `dev`."""
    if holder.device != dev:
        raise ValueError(f"tensors on one device are needed (GPU {dev}; those of a {type(holder).__name__} are not)")


def _rows(t, shape, dtype, what):
    """Stride between the tokens of a [tokens][heads][head_dim] tensor of dense rows (0: dense)."""
    if t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return 0
    st = t.stride()
    if t.dtype is dtype and t.shape == shape and st[2] == 1 and st[1] == shape[2]:
        if shape[0] < 2:
            return 0
        if st[0] >= shape[1] * shape[2]:  # (zero would mean dense)
            return st[0]
        raise ValueError(f"the rows of {what} overlap")
    if t.dtype is not dtype:
        raise TypeError(f"{what} is {t.dtype} beside a cache of {dtype}")
    if t.shape != shape:
        raise ValueError(f"{what} is {shape}")
    if t.numel() and (st[2] != 1 or shape[1] > 1):
        raise ValueError(f"{what} has dense rows")
    return _rows(t.as_strided(shape, (st[0], shape[2], 1)), shape, dtype, what) if t.numel() else 0


class Cache:
    """The pool of pages of one layer: k [pages][kv_heads][page_tokens][head_dim]
    and v [pages][kv_heads][head_dim][page_tokens], int8 or float8_e4m3fn, with
    their scales [pages][kv_heads] fp32; act_dtype: of queries, keys and values."""

    def __init__(self, k, v, k_scale, v_scale, act_dtype):
        pages, kv_heads, page_tokens, head_dim = k.shape
        if k.dtype not in _CODES or v.dtype is not k.dtype or act_dtype not in _ACTS:
            raise TypeError(f"a cache of {k.dtype} and {v.dtype} for {act_dtype}")
        if v.shape != (pages, kv_heads, head_dim, page_tokens):
            raise ValueError("v is [pages][kv_heads][head_dim][page_tokens]")
        for t in (k_scale, v_scale):
            if t.dtype is not torch.float32 or t.shape != (pages, kv_heads):
                raise ValueError("scales are [pages][kv_heads] fp32")
        if not all(t.is_contiguous() for t in (k, v, k_scale, v_scale)):
            raise ValueError("a cache's tensors are contiguous")
        self.k, self.v, self.k_scale, self.v_scale, self.act_dtype = k, v, k_scale, v_scale, act_dtype
        self.kv_heads, self.head_dim, self.page_tokens = kv_heads, head_dim, page_tokens
        devices = {t.get_device() for t in (k, v, k_scale, v_scale)}
        if len(devices) != 1:
            raise ValueError("a cache's tensors are on one device")
        self.device = devices.pop()
        self.c = _Cache(_CODES[k.dtype], _ACTS[act_dtype], kv_heads, head_dim, page_tokens, 0, pages,
                        k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())
        self._ref, self._at = ctypes.byref(self.c), ctypes.pointer(self.c)

    def tensors(self):
        return self.k, self.v, self.k_scale, self.v_scale


def new_cache(pages, kv_heads, page_tokens, head_dim, act_dtype, codes=torch.int8, device="cuda") -> Cache:
    """A cache of zeros, with the least scale."""
    k = torch.zeros((pages, kv_heads, page_tokens, head_dim), dtype=torch.uint8, device=device)
    v = torch.zeros((pages, kv_heads, head_dim, page_tokens), dtype=torch.uint8, device=device)
    ks, vs = (torch.full((pages, kv_heads), 2.0 ** -100, dtype=torch.float32, device=device) for _ in range(2))
    return Cache(k.view(codes), v.view(codes), ks, vs, act_dtype)


class Batch:
    """The requests of a step: their table rows [requests][width] int32 (rows of
    any stride), `tokens` rows of new tokens (padding included), no request with
    more than max_new of them. starts [requests + 1] and lens [requests] int32 are
    made here unless given (spear_kv_pages writes them)."""

    def __init__(self, table, tokens, max_new=None, starts=None, lens=None):
        if table.dtype is not torch.int32 or table.dim() != 2 or (table.numel() and table.stride(1) != 1):
            raise ValueError("table is [requests][width] int32 of dense rows")
        R, width = table.shape
        if R > 1 and table.stride(0) < width:
            raise ValueError("the rows of table overlap")

        def ints(t, n, what):
            t = torch.zeros(n, dtype=torch.int32, device=table.device) if t is None else t
            _ints(t, n, what)
            return t

        self.table, self.tokens, self.requests = table, _size(tokens, "tokens"), R
        self.starts, self.lens = ints(starts, R + 1, "starts"), ints(lens, R, "lens")
        self.max_new = max(1, self.tokens) if max_new is None else _size(max_new, "max_new")
        self.device = table.get_device()
        if self.starts.get_device() != self.device or self.lens.get_device() != self.device:
            raise ValueError("a batch's tensors are on one device")
        self.c = _Batch(R, self.tokens, self.max_new, width, _size(table.stride(0), "table's stride") if R > 1 else 0, 0,
                        self.starts.data_ptr(), self.lens.data_ptr(), table.data_ptr())
        self._ref = ctypes.byref(self.c)


def pages(batch: Batch, held, fresh, free_pages, slots, positions, taken, *, page_tokens, stream=None):
    """Block tables, slots and positions of a step (include/spear_kv.h)."""
    dev = _device_of(held, fresh, free_pages, slots, positions, taken)
    _on(batch, dev)
    R, T = batch.requests, batch.tokens
    a = _Pages(_size(page_tokens, "page_tokens"), free_pages.numel(), _ints(held, R, "held"), _ints(fresh, R, "fresh"),
               _ints(free_pages, free_pages.numel(), "free_pages"), _ints(slots, T, "slots"),
               _ints(positions, T, "positions"), _ints(taken, 2, "taken"))
    st = LIB.spear_kv_pages(batch._ref, ctypes.byref(a), _raw_stream(stream, dev))
    if st != 0:
        raise SpearError(st, "spear_kv_pages")


class Rope:
    """Rotary positions of the first rotary_dim features of a head; the frequencies
    as spear_rope_frequencies makes them, or given (int64 bits of 2^-64 turns)."""

    def __init__(self, rotary_dim, base=10000.0, *, interleaved=False, magnitude=1.0, factor=1.0,
                 context=0.0, low_turns=1.0, high_turns=4.0, freqs=None, device="cuda"):
        if freqs is None:
            freqs = torch.empty(max(0, rotary_dim) // 2, dtype=torch.int64)
            _check(LIB.spear_rope_frequencies(rotary_dim, base, factor, context, low_turns, high_turns,
                                              freqs.data_ptr()), "spear_rope_frequencies")
            freqs = freqs.to(device)
        if freqs.dtype is not torch.int64 or freqs.numel() != rotary_dim // 2 or not freqs.is_contiguous():
            raise ValueError("freqs is [rotary_dim / 2] int64")
        self.freqs, self.device = freqs, freqs.get_device()
        self.c = _Rope(rotary_dim, int(bool(interleaved)), magnitude, 0, freqs.data_ptr())


_NO_ROPE = _Rope(0, 0, 1.0, 0, None)


def append(cache: Cache, k, v, slots, positions=None, *, rope: Rope | None = None, q=None, q_out=None,
           stream=None):
    """New tokens into the cache, queries turned on the way (include/spear_kv.h):
    k, v [tokens][kv_heads][head_dim], q, q_out [tokens][heads][head_dim]."""
    dev = _device_of(k, v, slots, positions, q, q_out)
    _on(cache, dev)
    T, D, act = k.shape[0], cache.head_dim, cache.act_dtype
    kv = (T, cache.kv_heads, D)
    if (q is None) != (q_out is None) or (rope is not None and positions is None):
        raise ValueError("append: q and q_out go together, and a rotation takes positions")
    c = _NO_ROPE
    if rope is not None:
        c = rope.c
        if c.rotary_dim:
            _on(rope, dev)
    kl, vl = _rows(k, kv, act, "k"), _rows(v, kv, act, "v")
    at = None if positions is None else _ints(positions, T, "positions")
    if q is None:
        a = _Append(T, 0, None, k.data_ptr(), v.data_ptr(), None, 0, kl, vl, 0, _ints(slots, T, "slots"), at, c)
    else:
        qs = (T, q.shape[1], D)
        a = _Append(T, qs[1], q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr(), _rows(q, qs, act, "q"), kl,
                    vl, _rows(q_out, qs, act, "q_out"), _ints(slots, T, "slots"), at, c)
    st = LIB.spear_kv_append(cache._ref, ctypes.byref(a), _raw_stream(stream, dev))
    if st != 0:
        raise SpearError(st, "spear_kv_append")


def read(cache: Cache, slots, k_out, v_out, stream=None):
    """What the tokens at `slots` stand for: k_out, v_out [n][kv_heads][head_dim]."""
    dev = _device_of(slots, k_out, v_out)
    _on(cache, dev)
    n = slots.numel()
    for t, what in ((k_out, "k_out"), (v_out, "v_out")):
        if t.dtype is not cache.act_dtype or not t.is_contiguous() or t.numel() != n * cache.kv_heads * cache.head_dim:
            raise ValueError(f"read: {what} is [{n}][kv_heads][head_dim] in the activation dtype")
    st = LIB.spear_kv_read(cache._ref, n, _ints(slots, n, "slots"), k_out.data_ptr(), v_out.data_ptr(),
                           _raw_stream(stream, dev))
    if st != 0:
        raise SpearError(st, "spear_kv_read")


class AttentionPlan:
    """What the attention calls of a step share: the batch, the head counts, window
    and prefix [requests] int32, and the plan buffer that attention_plan writes."""

    def __init__(self, cache: Cache, batch: Batch, heads, *, window=0, prefix=None):
        self.cache, self.batch, self.heads, self.prefix = cache, batch, _size(heads, "heads"), prefix
        self.c = _Attention(ctypes.pointer(cache.c), ctypes.pointer(batch.c), self.heads, _size(window, "window"),
                            None if prefix is None else _ints(prefix, batch.requests, "prefix"))
        plan, work = ctypes.c_size_t(), ctypes.c_size_t()
        _check(LIB.spear_attention_sizes(ctypes.byref(self.c), ctypes.byref(plan), ctypes.byref(work)),
               "spear_attention_sizes")
        self.workspace_bytes = work.value
        self.buffer = torch.empty(plan.value, dtype=torch.uint8, device=batch.table.device)
        self.c.plan, self.c.plan_bytes = self.buffer.data_ptr(), plan.value
        self.device = batch.device
        if prefix is not None and prefix.get_device() != self.device:
            raise ValueError("a plan's tensors are on one device")
        self._batch = ctypes.pointer(batch.c)
        self._prefix = None if prefix is None else prefix.data_ptr()


def attention_workspace(plan: AttentionPlan) -> int:
    """Workspace bytes of the plan's attention calls (zero-filled once)."""
    return plan.workspace_bytes


def attention_plan(plan: AttentionPlan, stream=None):
    """Writes the plan from the batch's starts and lens, window and prefix."""
    dev = _device_of(plan.buffer)
    _on(plan.batch, dev)
    st = LIB.spear_attention_plan(ctypes.byref(plan.c), _raw_stream(stream, dev))
    if st != 0:
        raise SpearError(st, "spear_attention_plan")


def attention(plan: AttentionPlan, q, out, *, workspace, cache: Cache | None = None, scale=None, softcap=0.0,
              slopes=None, stream=None):
    """Attention of the batch's rows over the cache (the plan's own unless given:
    another layer's, of the same sizes): q, out [tokens][heads][head_dim]; scale
    1/sqrt(head_dim) unless given; slopes [heads] fp32."""
    own = plan.cache
    cache = own if cache is None else cache
    dev = _device_of(q, out, workspace, slopes)
    _on(plan, dev)
    _on(cache, dev)
    D, heads = cache.head_dim, plan.heads
    if cache is not own and (cache.kv_heads, D, cache.page_tokens) != (own.kv_heads, own.head_dim, own.page_tokens):
        raise ValueError("attention: a cache of the plan's sizes")
    if slopes is not None and (slopes.dtype is not torch.float32 or slopes.numel() != heads or not slopes.is_contiguous()):
        raise ValueError("attention: slopes is [heads] fp32")
    shape, act = (plan.batch.tokens, heads, D), cache.act_dtype
    a = _Attention(cache._at, plan._batch, heads, plan.c.window, plan._prefix, plan.c.plan,
                   plan.c.plan_bytes, q.data_ptr(), out.data_ptr(), _rows(q, shape, act, "q"), _rows(out, shape, act, "out"),
                   None if slopes is None else slopes.data_ptr(), D ** -0.5 if scale is None else scale, softcap,
                   workspace.data_ptr(), workspace.numel() * workspace.element_size())
    st = LIB.spear_attention(ctypes.byref(a), _raw_stream(stream, dev))
    if st != 0:
        raise SpearError(st, "spear_attention")
    return out
