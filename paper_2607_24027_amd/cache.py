"""ctypes binding of the serving operators (C ABI in include/sol_cache.h).

Argument marshalling only, as in ``binding``: torch tensors supply device memory and the current stream, every step of
the computation runs in the library's HIP kernels.  A step of autoregressive generation for a ragged batch::

    new = cache.tables(lens, add, table, ring, state, rows)
    q, k = cache.qk_norm_rope(q, k, q_weight, k_weight, cos, sin, new.positions[None])
    cache.append(k[0], v, store, new.slots)
    out = cache.forward(q[0], store, table, new.lens, new.row_start, new.positions)

Tensors of tokens are heads first ([B, H, N, d], [H, T, d]) with any strides as long as the channels of a head are
contiguous: pass the projection's output through ``transpose`` and it is read where it is.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import NamedTuple, Optional

from . import binding as _b

PAGE = 64
HALVES, PAIRS = 0, 1

_P, _I, _F, _S = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
# (restype, argtypes) for every symbol of include/sol_cache.h
SIGNATURES = {
    "sol_qk_norm_rope": (_I, [_P] * 13 + [_I] * 8 + [_F, _I, _I, _P]),
    "sol_cache_tables": (_I, [_P] * 10 + [_I] * 4 + [_P]),
    "sol_cache_append": (_I, [_P] * 6 + [_I] * 5 + [_P]),
    "sol_cache_read": (_I, [_P] * 6 + [_I] * 5 + [_P]),
    "sol_cache_bytes": (_S, [_I] * 3),
    "sol_cache_workspace_bytes": (_S, [_I] * 7),
    "sol_cache_forward": (_I, [_P] * 9 + [_I] * 10 + [_P, _S, _P]),
}
_INVALID = ctypes.c_size_t(-1).value

_lib = None


def lib() -> ctypes.CDLL:
    """libsolattn.so with the signatures of this module (raises if it has not been built)."""
    global _lib
    if _lib is None:
        handle = _b.lib()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def _on(device):
    """The library launches on the current device: makes it the tensors' one for the call."""
    import torch
    if device.index is None or torch.cuda.current_device() == device.index:
        return contextlib.nullcontext()
    return torch.cuda.device(device)


def _strides(t):
    """Strides of all dimensions but the last, as a C array (of a dimension of one element: 0)."""
    s = [st if n > 1 else 0 for st, n in zip(t.stride()[:-1], t.shape[:-1])]
    return (ctypes.c_longlong * len(s))(*s)


def _ref(arr):
    return None if arr is None else ctypes.cast(arr, _P)


def _check_heads(name, t, dim, ref=None, writable=False):
    if t.dim() != dim:
        raise ValueError(f"{name} must have {dim} dimensions (got {tuple(t.shape)})")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"the channels of {name} must be contiguous")
    _b._dtype_code(t)
    if ref is not None:
        if t.dtype != ref.dtype:
            raise ValueError(f"{name} must have dtype {ref.dtype} (got {t.dtype})")
        if t.device != ref.device:
            raise ValueError(f"{name} must be on {ref.device} (got {t.device})")
    if writable:
        rows = sorted((st, n) for st, n in zip(t.stride()[:-1], t.shape[:-1]) if n > 1)
        reach = t.shape[-1]
        for st, n in rows:
            if st < reach:
                raise ValueError(f"rows of {name} overlap")
            reach = st * (n - 1) + reach


def _check_ints(name, t, shape, device):
    import torch
    _b._check_buffer(name, t, shape, (torch.int32,), device)


def _overlap(a, b):
    """Whether two tensors share memory, by their outermost bytes: False, or True where they may."""
    if a.device != b.device or not a.numel() or not b.numel():
        return False

    def span(t):
        last = sum(st * (n - 1) for st, n in zip(t.stride(), t.shape))
        return t.data_ptr(), t.data_ptr() + (last + 1) * t.element_size()
    (a0, a1), (b0, b1) = span(a), span(b)
    return a0 < b1 and b0 < a1


def _disjoint(name, t, **others):
    for other, o in others.items():
        if o is not None and t is not None and _overlap(t, o):
            raise ValueError(f"{name} must not overlap {other}")


def qk_norm_rope(q, k, q_weight=None, k_weight=None, cos=None, sin=None, positions=None, eps: float = 1e-6,
                 interleaved: bool = False, q_out=None, k_out=None):
    """RMS norm of each head of q [B,Hq,N,d] and k [B,Hk,N,d] (either may be None) and the rotation by position, in one pass.

    q_weight, k_weight: [d] (bf16 or f32, one dtype) or None for ones.  cos, sin: f32 [P, rot / 2] tables (None: no rotation)
    whose row is the token's position; positions: int32 [B, N], or None for 0 ... N - 1.  Tokens whose position is not a
    row of the tables are left out (their rows of given outputs stay as they were, those of new ones are undefined).
    interleaved: channels 2i and 2i + 1 are a pair, otherwise i and i + rot / 2.  q_out, k_out: any strides; new contiguous
    tensors by default, as forward() takes them.  Returns (q_out, k_out)."""
    import torch
    ref = q if q is not None else k
    if ref is None:
        raise ValueError("one of q and k must be given")
    given = {"q": (q, q_weight, q_out), "k": (k, k_weight, k_out)}
    B, _, N, d = ref.shape if ref.dim() == 4 else (0, 0, 0, 0)
    wdtype = None
    outs, sin_, sout = {}, {}, {}
    for name, (x, w, out) in given.items():
        outs[name], sin_[name], sout[name] = None, None, None
        if x is None:
            if w is not None or out is not None:
                raise ValueError(f"{name}_weight and {name}_out need {name}")
            continue
        _check_heads(name, x, 4, ref)
        if (x.shape[0], x.shape[2], x.shape[3]) != (B, N, d):
            raise ValueError(f"q and k must agree in B, N and d (got {tuple(x.shape)} for {name})")
        if w is not None:
            _b._check_buffer(f"{name}_weight", w, (d,), (torch.bfloat16, torch.float32), x.device)
            if wdtype is not None and w.dtype != wdtype:
                raise ValueError("q_weight and k_weight must have one dtype")
            wdtype = w.dtype
        if out is not None:
            if tuple(out.shape) != tuple(x.shape):
                raise ValueError(f"{name}_out must have shape {tuple(x.shape)} (got {tuple(out.shape)})")
            _check_heads(f"{name}_out", out, 4, x, writable=True)
    for name, (x, w, out) in given.items():
        _disjoint(f"{name}_out", out, q=q, k=k, cos=cos, sin=sin, positions=positions, q_weight=q_weight, k_weight=k_weight)
    _disjoint("q_out", q_out, k_out=k_out)
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin must be given together")
    P = rot = 0
    if cos is not None:
        if cos.dim() != 2:
            raise ValueError("cos and sin must be [P, rot / 2]")
        P, rot = cos.shape[0], 2 * cos.shape[1]
        for name, t in (("cos", cos), ("sin", sin)):
            _b._check_buffer(name, t, cos.shape, (torch.float32,), ref.device)
    if positions is not None:
        _check_ints("positions", positions, (B, N), ref.device)
    _b._require_gpu(ref)
    for name, (x, w, out) in given.items():
        if x is not None:
            outs[name] = out if out is not None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
            sin_[name], sout[name] = _strides(x), _strides(outs[name])
    with _on(ref.device):
        _b._check(lib().sol_qk_norm_rope(
            _b._ptr(q), _b._ptr(k), _b._ptr(outs["q"]), _b._ptr(outs["k"]), _ref(sin_["q"]), _ref(sin_["k"]),
            _ref(sout["q"]), _ref(sout["k"]), _b._ptr(q_weight), _b._ptr(k_weight), _b._ptr(cos), _b._ptr(sin),
            _b._ptr(positions), B, 0 if q is None else q.shape[1], 0 if k is None else k.shape[1], N, d, P, rot,
            PAIRS if interleaved else HALVES, float(eps), _b._dtype_code(ref),
            _b.SOL_F32 if wdtype == torch.float32 else _b.SOL_BF16, _b._stream(ref.device)))
    return outs["q"], outs["k"]


class Step(NamedTuple):
    """What tables() gives: row_start [S + 1], slots and positions [rows], lens [S] and state [2] after the step."""
    row_start: "object"
    slots: "object"
    positions: "object"
    lens: "object"
    state: "object"


def tables(lens, add, table, ring, state, rows: int, out: Optional[Step] = None) -> Step:
    """Pages, slots and positions of one step: int32 lens [S] (tokens held), add [S] (tokens to add, or below 0 to take
    back), table [S, max_pages] and ring [P] (both updated), state [2] (place and number of the free pages in the ring);
    rows: the rows of slots and positions to fill, at least the sum of the positive adds.  The rules are in
    include/sol_cache.h.  out: tensors of an earlier step to write into (not lens and state themselves)."""
    import torch
    if lens.dim() != 1 or table.dim() != 2 or ring.dim() != 1:
        raise ValueError("lens, table and ring must be [S], [S, max_pages] and [P]")
    S, MP = lens.shape[0], table.shape[1]
    for name, t, shape in (("lens", lens, (S,)), ("add", add, (S,)), ("table", table, (S, MP)), ("ring", ring, ring.shape),
                           ("state", state, (2,))):
        _check_ints(name, t, shape, lens.device)
    if rows < 0:
        raise ValueError(f"rows must not be negative (got {rows})")
    shapes = {"row_start": (S + 1,), "slots": (rows,), "positions": (rows,), "lens": (S,), "state": (2,)}
    if out is not None:
        for name, shape in shapes.items():
            _check_ints(f"out.{name}", getattr(out, name), shape, lens.device)
        for name in shapes:
            _disjoint(f"out.{name}", getattr(out, name), lens=lens, add=add, table=table, ring=ring, state=state,
                      **{f"out.{o}": getattr(out, o) for o in shapes if o != name})
    _disjoint("table", table, lens=lens, add=add, ring=ring, state=state)
    _disjoint("ring", ring, lens=lens, add=add, state=state)
    _b._require_gpu(lens)
    if out is None:
        # one allocation, each part on 16 bytes
        sizes = [-(-n // 4) * 4 for n in (S + 1, rows, rows, S, 2)]
        flat = torch.empty(sum(sizes), dtype=torch.int32, device=lens.device)
        parts, at = [], 0
        for n, size in zip((S + 1, rows, rows, S, 2), sizes):
            parts.append(flat[at:at + n])
            at += size
        out = Step(*parts)
    with _on(lens.device):
        _b._check(lib().sol_cache_tables(_b._ptr(lens), _b._ptr(add), _b._ptr(table), _b._ptr(ring), _b._ptr(state),
                                         _b._ptr(out.lens), _b._ptr(out.state), _b._ptr(out.row_start), _b._ptr(out.slots),
                                         _b._ptr(out.positions), S, MP, ring.shape[0], rows, _b._stream(lens.device)))
    return out


def cache_bytes(pages: int, heads: int, d: int) -> int:
    """Bytes of a store of that many pages (of 64 tokens) and key/value heads."""
    n = int(lib().sol_cache_bytes(pages, heads, d))
    if n == _INVALID:
        raise ValueError(f"no store of {pages} pages, {heads} heads of {d} channels")
    return n


def empty(pages: int, heads: int, d: int, device):
    """A store [pages, heads, 68 d] of bytes for append(); its contents are undefined."""
    import torch
    cache_bytes(pages, heads, d)
    return torch.empty((pages, heads, 68 * d), dtype=torch.uint8, device=device)


def _check_store(store, device=None):
    """(pages, heads, d) of a store."""
    import torch
    if store.dim() != 3 or store.shape[2] not in (68 * 64, 68 * 128):
        raise ValueError(f"store must be [pages, heads, 68 d] bytes with d = 64 or 128 (got {tuple(store.shape)})")
    _b._check_buffer("store", store, store.shape, (torch.uint8,), store.device if device is None else device)
    return store.shape[0], store.shape[1], store.shape[2] // 68


def append(k, v, store, slots):
    """Writes k, v [heads, T, d] into the slots (int32 [T], slot = 64 page + token; others are left out) of the store."""
    P, H, d = _check_store(store)
    _check_heads("k", k, 3)
    _check_heads("v", v, 3, k)
    if tuple(k.shape) != tuple(v.shape):
        raise ValueError(f"k and v must have one shape (got {tuple(k.shape)} and {tuple(v.shape)})")
    if (k.shape[0], k.shape[2]) != (H, d):
        raise ValueError(f"k and v must have {H} heads of {d} channels as the store has (got {tuple(k.shape)})")
    _check_store(store, k.device)
    T = k.shape[1]
    _check_ints("slots", slots, (T,), k.device)
    _disjoint("store", store, k=k, v=v, slots=slots)
    _b._require_gpu(k)
    ks, vs = _strides(k), _strides(v)
    with _on(k.device):
        _b._check(lib().sol_cache_append(_b._ptr(k), _b._ptr(v), _ref(ks), _ref(vs), _b._ptr(store), _b._ptr(slots), T, H, d,
                                         P, _b._dtype_code(k), _b._stream(k.device)))


def read(store, slots, dtype=None, k_out=None, v_out=None):
    """(k, v) [heads, T, d] of the slots (int32 [T]), as the values that their codes stand for; zeros for slots outside the
    store.  dtype: bf16 (default) or f32.  With k_out or v_out given, only what is given is read."""
    import torch
    P, H, d = _check_store(store)
    if slots.dim() != 1:
        raise ValueError("slots must be [T]")
    T = slots.shape[0]
    _check_ints("slots", slots, (T,), store.device)
    given = [t for t in (k_out, v_out) if t is not None]
    if given:
        if dtype is not None and dtype != given[0].dtype:
            raise ValueError(f"dtype is {dtype}, that of the outputs {given[0].dtype}")
        for name, t in (("k_out", k_out), ("v_out", v_out)):
            if t is None:
                continue
            _check_heads(name, t, 3, given[0], writable=True)
            if tuple(t.shape) != (H, T, d):
                raise ValueError(f"{name} must have shape {(H, T, d)} (got {tuple(t.shape)})")
            if t.device != store.device:
                raise ValueError(f"{name} must be on {store.device} (got {t.device})")
            _disjoint(name, t, store=store, slots=slots)
        _disjoint("k_out", k_out, v_out=v_out)
    dt = given[0].dtype if given else torch.bfloat16 if dtype is None else dtype
    if dt not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dt}")
    _b._require_gpu(store)
    if not given:
        k_out, v_out = torch.empty((2, H, T, d), dtype=dt, device=store.device).unbind(0)
    ks, vs = (None if t is None else _strides(t) for t in (k_out, v_out))
    with _on(store.device):
        _b._check(lib().sol_cache_read(_b._ptr(store), _b._ptr(slots), _b._ptr(k_out), _b._ptr(v_out), _ref(ks), _ref(vs), T,
                                       H, d, P, _b.SOL_BF16 if dt == torch.bfloat16 else _b.SOL_F32, _b._stream(store.device)))
    return k_out, v_out


def workspace_bytes(S: int, T: int, max_rows: int, Hq: int, Hk: int, d: int, max_pages: int) -> int:
    """Scratch bytes of forward() for S requests with T rows in all, max_rows of one at most."""
    n = int(lib().sol_cache_workspace_bytes(S, T, max_rows, Hq, Hk, d, max_pages))
    if n == _INVALID:
        raise ValueError(_b.last_error())
    return n


def forward(q, store, table, lens, row_start, positions, causal_granule: int = 1, max_rows: Optional[int] = None, out=None,
            workspace=None):
    """Attention of the rows q [Hq, T, d] of S requests over their tokens in the store.

    table [S, max_pages], lens [S] (with the new tokens), row_start [S + 1], positions [T]: int32, as tables() gives them.
    causal_granule: 1 is token-causal, the tokens of a frame frame-causal, the longest length or more no mask.  max_rows:
    rows of the request that has most (default T: any).  out: like q, any strides; by default with q's order of
    dimensions in memory, rows outside the requests undefined.  workspace: 1-D uint8 tensor of workspace_bytes(...)
    bytes, by default a new one of torch's allocator (inside a graph capture: of the graph's own pool).  Returns out."""
    import torch
    P, Hk, d = _check_store(store)
    _check_heads("q", q, 3)
    Hq, T = q.shape[0], q.shape[1]
    if q.shape[2] != d:
        raise ValueError(f"q must have {d} channels as the store has (got {q.shape[2]})")
    _check_store(store, q.device)
    if lens.dim() != 1 or table.dim() != 2:
        raise ValueError("lens and table must be [S] and [S, max_pages]")
    S, MP = lens.shape[0], table.shape[1]
    for name, t, shape in (("lens", lens, (S,)), ("table", table, (S, MP)), ("row_start", row_start, (S + 1,)),
                           ("positions", positions, (T,))):
        _check_ints(name, t, shape, q.device)
    if out is not None:
        if tuple(out.shape) != tuple(q.shape):
            raise ValueError(f"out must have shape {tuple(q.shape)} (got {tuple(out.shape)})")
        _check_heads("out", out, 3, q, writable=True)
        _disjoint("out", out, q=q, store=store, table=table, lens=lens, row_start=row_start, positions=positions,
                  workspace=workspace)
    if workspace is not None:
        if workspace.dim() != 1:
            raise ValueError("workspace must be a 1-D uint8 tensor")
        _b._check_buffer("workspace", workspace, workspace.shape, (torch.uint8,), q.device)
        _disjoint("workspace", workspace, q=q, store=store, table=table, lens=lens, row_start=row_start, positions=positions)
    _b._require_gpu(q)
    rows = T if max_rows is None else int(max_rows)
    if workspace is None:
        need = int(lib().sol_cache_workspace_bytes(S, T, rows, Hq, Hk, d, MP))
        if need != _INVALID and need:   # invalid arguments are the call's to report
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    if out is None:
        out = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device) if _dense(q) else torch.empty_like(q)
    qs, os_ = _strides(q), _strides(out)
    with _on(q.device):
        _b._check(lib().sol_cache_forward(
            _b._ptr(q), _ref(qs), _b._ptr(out), _ref(os_), _b._ptr(store), _b._ptr(table), _b._ptr(lens),
            _b._ptr(row_start), _b._ptr(positions), S, T, rows, Hq, Hk, d, P, MP, int(causal_granule), _b._dtype_code(q),
            _b._ptr(workspace), 0 if workspace is None else workspace.numel(), _b._stream(q.device)))
    return out


def _dense(t):
    """Whether t fills its memory without holes or overlaps."""
    reach = 1
    for st, n in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n > 1):
        if st != reach:
            return False
        reach *= n
    return True
